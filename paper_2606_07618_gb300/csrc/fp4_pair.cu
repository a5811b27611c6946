// Products of many tokens: a pair of CTAs (cta_group::2) forms 256 tokens by 256 columns
// (gated: 128 gate and the same 128 up columns) and walks several such tiles.
//
//   out[t][n] = epilogue( sum_k q[t][k] p[n][k] )
//
// Tokens are the MMA's M side, so a thread's accumulator columns are consecutive columns of
// one row: a block of 32 for MXFP4 is one thread's, and stores go out as boxes.  Each CTA
// loads its 128 token rows and half of the 256 weight rows; the leader's MMA reads both halves,
// so a stage of K costs 64 KB of loads for 256 x 256 x 128 bytes of K.
//   warp 8   loads: 128 bytes of K a stage, operands and scale atoms, by TMA; completion is
//            counted on the leader's barrier
//   warp 9   (leader) copies the scale atoms of both CTAs to tensor memory and issues the MMAs
//   warps 0-7  accumulators to results, 32 columns at a time, through two 2 KB boxes of shared
//            memory a warp, stored by TMA (rows of single elements where the result's
//            stride does not allow that); beside the next tile's MMAs
//
// Tensor memory holds two accumulators of 256 columns and 48 columns of scales in 512: with
// scales the accumulators overlap in 48 columns, which the epilogue drains first.  An arrival
// of every epilogue warp a tile ("drained", a barrier for even and one for odd tiles, as a warp
// may be a tile ahead of another) says that it is done with the tile before and has read
// the overlapping columns of this one; the next tile's MMAs wait for all of them.
//
// Waits are bounded as in fp4_gemm.cu.
#include "fp4_tile.cuh"

namespace nvfp4 {
namespace mm {
namespace {

constexpr int kEpiWarps = 8;
constexpr int kThreadsPair = (kEpiWarps + 2) * 32;
constexpr int kBox = 2048;                                   // 32 rows of 64 bytes
constexpr int kPairStages = 6;                               // at most

struct PairParams {
    CUtensorMap p, p2, q, sp, sp2, sq;
    CUtensorMap o, o2, o3;                                   // results: D or h; dg and du
    int64_t k;
    int tiles_t, tiles_n;
    int64_t boxed;                                           // columns of D or h that go out by TMA
    Epilogue e;
};

template <int KIND>
struct Pair {
    static constexpr int kOp = 128 * kRow;                   // a CTA's part of an operand: 16 KB
    static constexpr int kS = atoms(KIND) * kAtom;
    static constexpr int kStage = 2 * kOp + 3 * kS;          // + scales of its tokens, of all columns
    static constexpr int kStages = KIND == kBf16 ? 6 : 5;
    static constexpr int kSmem = kStages * kStage + kEpiWarps * 2 * kBox + 1024;
    static constexpr int kSf = 464;                          // scale columns: tokens, then columns
    static constexpr int kAcc1 = KIND == kBf16 ? 256 : 208;  // the second accumulator
};

__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}
// Arrives on this barrier of both CTAs once the MMAs issued so far have finished.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void store_wait_read1() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }

// Tile number -> token and column tile.  Eight token tiles are walked for each column tile, so
// that the tiles in flight at one time cover a near-square of the result.
__device__ __forceinline__ void tile_at(int i, int tiles_t, int tiles_n, int& tt, int& tn) {
    const int per = 8 * tiles_n, g = i / per, first = 8 * g, rows = min(8, tiles_t - first), j = i - g * per;
    tt = first + j % rows;
    tn = j / rows;
}

// A warp's boxes: 32 rows (lanes) of 64 bytes, 64-byte swizzle.
struct Boxes {
    uint8_t* base;
    int next = 0;
    int lane;
    __device__ __forceinline__ uint8_t* take() {             // the box of two stores ago has been read
        if (lane == 0) store_wait_read1();
        __syncwarp();
        return base + (next++ & 1) * kBox;
    }
    __device__ __forceinline__ void put(uint8_t* box, int c, uint4 v) const {
        *reinterpret_cast<uint4*>(box + lane * 64 + ((c ^ (lane >> 1 & 3)) << 4)) = v;
    }
    __device__ __forceinline__ void store(const uint8_t* box, const CUtensorMap* map, int64_t n, int64_t t) const {
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
            tma_store_2d(map, (int)n, (int)t, smem_u32(box));
            tma_store_commit();
        }
    }
    // the same by single elements of ES bytes: rows t.. below T, columns n.. below N
    template <int ES>
    __device__ __forceinline__ void spill(const uint8_t* box, void* out, int64_t ld, int64_t n, int64_t t, int64_t N,
                                          int64_t T) const {
        __syncwarp();
        for (int r = lane >> 4; r < 32; r += 2) {
            const int w = lane & 15;
            const uint32_t v = *reinterpret_cast<const uint32_t*>(box + r * 64 + (((w >> 2) ^ (r >> 1 & 3)) << 4) + (w & 3) * 4);
            if (t + r >= T) continue;
            if (ES == 4) {
                if (n + w < N) static_cast<uint32_t*>(out)[(t + r) * ld + n + w] = v;
            } else {
                if (n + 2 * w < N) static_cast<uint16_t*>(out)[(t + r) * ld + n + 2 * w] = (uint16_t)v;
                if (n + 2 * w + 1 < N) static_cast<uint16_t*>(out)[(t + r) * ld + n + 2 * w + 1] = (uint16_t)(v >> 16);
            }
        }
        __syncwarp();
    }
};

__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// 32 bf16 (16 words) of this lane's row to a box and out; columns from `boxed` on by elements.
__device__ __forceinline__ void out_bf16(Boxes& bx, const uint32_t (&w)[16], int64_t boxed, const CUtensorMap* map, void* out,
                                         int64_t ld, int64_t n, int64_t t, int64_t N, int64_t T) {
    if (n >= N || t >= T) return;                            // uniform: t is the warp's first row
    uint8_t* box = bx.take();
#pragma unroll
    for (int c = 0; c < 4; c++) bx.put(box, c, make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]));
    if (n < boxed)
        bx.store(box, map, n, t);
    else
        bx.spill<2>(box, out, ld, n, t, N, T);
}

template <int KIND, int MODE>
__global__ void __launch_bounds__(kThreadsPair, 1) __cluster_dims__(2, 1, 1) pair_kernel(const __grid_constant__ PairParams P) {
    using C = Pair<KIND>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kPairStages + 4];
    __shared__ int s_abort;
    __shared__ uint32_t s_tmem;
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
    const uint32_t rank = cluster_rank();
    const int nst = (int)((P.k + stage_k(KIND) - 1) / stage_k(KIND));
    const int ntiles = P.tiles_t * P.tiles_n, step = (int)gridDim.x / 2, first = (int)blockIdx.x / 2;
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kPairStages, accf0 = empty0 + 8 * kPairStages,
                   drained0 = accf0 + 16;

    if (tid == 0) {
        for (int b = 0; b < C::kStages; b++) {
            mbar_init(full0 + 8 * b, 1);
            mbar_init(empty0 + 8 * b, 1);
        }
        mbar_init(accf0, 1);
        mbar_init(accf0 + 8, 1);
        mbar_init(drained0, 2 * kEpiWarps);
        mbar_init(drained0 + 8, 2 * kEpiWarps);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kEpiWarps + 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_barrier();                                       // both CTAs' barriers and tensor memory are there
    tc_fence_after();
    grid_launch_dependents();
    grid_dependency_wait();
    const uint32_t tmem = s_tmem;

    if (warp == kEpiWarps) {
        Ring ring;
        const uint32_t leader_full = at_rank(full0, 0);
        bool ok = true;
        int issued = 0;
        for (int i = first; ok && i < ntiles; i += step) {
            int tt, tn;
            tile_at(i, P.tiles_t, P.tiles_n, tt, tn);
            const int t0 = tt * 256 + (int)rank * 128;
            for (int kc = 0; kc < nst; kc++) {
                const int r = ring.slot;
                if (issued >= C::kStages && !mbar_wait_warp(empty0 + 8 * r, ring.parity ^ 1)) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    const uint32_t st = smem_u32(base) + r * C::kStage, bar = leader_full + 8 * r;
                    if (rank == 0) mbar_expect_tx(full0 + 8 * r, 2 * C::kStage);
                    const int x = kc * (KIND == kBf16 ? 64 : 128);
                    tma_load_2d_pair(st, &P.q, x, t0, bar);
                    if (MODE == kPlain)
                        tma_load_2d_pair(st + C::kOp, &P.p, x, tn * 256 + (int)rank * 128, bar);
                    else
                        tma_load_2d_pair(st + C::kOp, rank == 0 ? &P.p : &P.p2, x, tn * 128, bar);
                    if (KIND != kBf16) {
                        const uint32_t sf = st + 2 * C::kOp;
                        const int a = kc * atoms(KIND);
                        tma_load_3d_pair(sf, &P.sq, 0, a, t0 >> 7, bar);
                        tma_load_3d_pair(sf + C::kS, &P.sp, 0, a, MODE == kPlain ? 2 * tn : tn, bar);
                        if (MODE == kPlain)
                            tma_load_3d_pair(sf + 2 * C::kS, &P.sp, 0, a, 2 * tn + 1, bar);
                        else
                            tma_load_3d_pair(sf + 2 * C::kS, &P.sp2, 0, a, tn, bar);
                    }
                }
                __syncwarp();
                if (issued < C::kStages) issued++;
                ring.next(C::kStages);
            }
        }
        // every slot in use read, hence landed
        if (issued < C::kStages) ring = Ring{0, 1};          // each used once
        for (int j = 0; ok && j < issued; j++, ring.next(C::kStages)) ok = mbar_wait_warp(empty0 + 8 * ring.slot, ring.parity ^ 1);
        if (!ok && lane == 0) atomicOr(&s_abort, 1);
    } else if (warp == kEpiWarps + 1 && rank == 0) {
        constexpr uint32_t id = idesc(KIND, 256, 256);
        Ring ring;
        int it = 0;
        bool ok = true;
        for (int i = first; ok && i < ntiles; i += step, it++) {
            if (it > 0 && !mbar_wait_warp(drained0 + 8 * ((it - 1) & 1), ((it - 1) >> 1) & 1)) ok = false;
            tc_fence_after();
            const uint32_t acc = tmem + (it & 1) * C::kAcc1;
            for (int kc = 0; ok && kc < nst; kc++) {
                const int r = ring.slot;
                if (!mbar_wait_warp(full0 + 8 * r, ring.parity)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t st = smem_u32(base) + r * C::kStage, sf = st + 2 * C::kOp;
#pragma unroll
                    for (int a = 0; a < atoms(KIND); a++) {
                        cp_atom<2>(tmem + C::kSf + 4 * a, atom_desc(sf + a * kAtom));
                        cp_atom<2>(tmem + C::kSf + 16 + 8 * a, atom_desc(sf + C::kS + a * kAtom));
                        cp_atom<2>(tmem + C::kSf + 16 + 8 * a + 4, atom_desc(sf + 2 * C::kS + a * kAtom));
                    }
                    const int left = (int)((P.k - (int64_t)kc * stage_k(KIND) + mma_k(KIND) - 1) / mma_k(KIND));
#pragma unroll
                    for (int kk = 0; kk < 4; kk++) {
                        if (kk >= left) break;
                        const int a = KIND == kNvfp4 ? kk : kk >> 1;
                        mma<KIND, 2>(acc, smem_desc(st + kk * 32, 16, 1024), smem_desc(st + C::kOp + kk * 32, 16, 1024),
                                     KIND == kMxfp4 ? id | sf_id(2 * (kk & 1)) : id, (uint32_t)(kc | kk), tmem + C::kSf + 4 * a,
                                     tmem + C::kSf + 16 + 8 * a);
                    }
                    commit_pair(empty0 + 8 * r);
                    if (kc == nst - 1) commit_pair(accf0 + 8 * (it & 1));
                }
                __syncwarp();
                ring.next(C::kStages);
            }
        }
        if (!ok && lane == 0) atomicOr(&s_abort, 1);
    } else if (warp < kEpiWarps) {
        const Epilogue& e = P.e;
        const float sp = scale_or_1(e.s_p), sp2 = MODE != kPlain ? scale_or_1(e.s_p2) : 1.0f, sq = scale_or_1(e.s_q);
        const int half = warp >> 2, q = warp & 3;
        Boxes bx{base + C::kStages * C::kStage + warp * 2 * kBox, 0, lane};
        const uint32_t leader_drained = at_rank(drained0, 0);
        bool bad = false;
        int it = 0;
        for (int i = first; i < ntiles; i += step, it++) {
            int tt, tn;
            tile_at(i, P.tiles_t, P.tiles_n, tt, tn);
            const int b = it & 1;
            const bool overlap = KIND != kBf16 && half == 1 - b;     // this warp reads the overlapping columns
            auto release = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at(leader_drained + 8 * b);
            };
            if (!overlap) release();                         // done with the tile before
            if (!mbar_wait(accf0 + 8 * b, (it >> 1) & 1)) {
                atomicOr(&s_abort, 1);
                break;
            }
            tc_fence_after();
            __syncwarp();
            const uint32_t acc = tmem + b * C::kAcc1 + ((uint32_t)(32 * q) << 16);
            const int64_t tw = (int64_t)tt * 256 + rank * 128 + 32 * q, t = tw + lane;   // the warp's first row, this lane's
            if (MODE == kPlain) {
#pragma unroll 1
                for (int c = 0; c < 4; c++) {
                    const int col = 128 * half + 32 * (overlap && half == 1 ? 3 - c : c);   // overlapping columns first
                    float v[32];
                    tmem_ld32(acc + col, v);
                    tmem_wait32(v);
                    if (overlap && c == 1) release();
                    const int64_t n = (int64_t)tn * 256 + col;
#pragma unroll
                    for (int j = 0; j < 32; j++) v[j] = v[j] * sp * sq;
                    if (e.out_f32) {
#pragma unroll
                        for (int g = 0; g < 2; g++) {
                            if (n + 16 * g >= e.N || tw >= e.T) continue;
                            uint8_t* box = bx.take();
#pragma unroll
                            for (int j = 0; j < 4; j++)
                                bx.put(box, j, make_uint4(__float_as_uint(v[16 * g + 4 * j]), __float_as_uint(v[16 * g + 4 * j + 1]),
                                                          __float_as_uint(v[16 * g + 4 * j + 2]), __float_as_uint(v[16 * g + 4 * j + 3])));
                            if (n + 16 * g < P.boxed)
                                bx.store(box, &P.o, n + 16 * g, tw);
                            else
                                bx.spill<4>(box, e.out, e.ldo, n + 16 * g, tw, e.N, e.T);
                        }
                    } else {
                        uint32_t w[16];
#pragma unroll
                        for (int j = 0; j < 16; j++) w[j] = pack2_bf16(v[2 * j], v[2 * j + 1]);
                        out_bf16(bx, w, P.boxed, &P.o, e.out, e.ldo, n, tw, e.N, e.T);
                    }
                }
            } else {
                float first_[2][32];                         // what overlaps: the up columns of the upper half, the gate's of the lower
                const int pre = half == 1 ? 128 : 0;
                tmem_ld32(acc + pre + 64 * half, first_[0]);
                tmem_ld32(acc + pre + 64 * half + 32, first_[1]);
                tmem_wait32(first_[0]);
                tmem_wait32(first_[1]);
                if (overlap) release();
                uint32_t sf2 = 0;
#pragma unroll
                for (int c = 0; c < 2; c++) {
                    float g[32], u[32], other[32];
                    tmem_ld32(acc + (128 - pre) + 64 * half + 32 * c, other);
                    const int64_t n = (int64_t)tn * 128 + 64 * half + 32 * c;
                    const bool row = t < e.T;
                    uint32_t dhw[16];
                    if (MODE == kGatedGrad) {
                        const uint16_t* at = e.dh + t * e.lddh + n;
                        if (row && n + 32 <= e.N && ((reinterpret_cast<uintptr_t>(at) & 15) == 0)) {
#pragma unroll
                            for (int j = 0; j < 4; j++) {
                                const uint4 d = *reinterpret_cast<const uint4*>(at + 8 * j);
                                dhw[4 * j] = d.x, dhw[4 * j + 1] = d.y, dhw[4 * j + 2] = d.z, dhw[4 * j + 3] = d.w;
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; j++) {
                                const uint32_t lo = row && n + 2 * j < e.N ? at[2 * j] : 0, hi = row && n + 2 * j + 1 < e.N ? at[2 * j + 1] : 0;
                                dhw[j] = lo | hi << 16;
                            }
                        }
                    }
                    tmem_wait32(other);
#pragma unroll
                    for (int j = 0; j < 32; j++) {
                        g[j] = (half == 1 ? other[j] : first_[c][j]) * sp * sq;
                        u[j] = (half == 1 ? first_[c][j] : other[j]) * sp2 * sq;
                    }
                    uint32_t hw[16];
                    if (MODE == kGated) {
                        float unused;
#pragma unroll
                        for (int j = 0; j < 16; j++)
                            hw[j] = pack2_bf16(activate<false>(e.act, g[2 * j], unused) * u[2 * j],
                                               activate<false>(e.act, g[2 * j + 1], unused) * u[2 * j + 1]);
                    } else {
                        uint32_t gs[16], us[16], gt[16], ut[16];
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            float dg[2], du[2], hv[2];
#pragma unroll
                            for (int z = 0; z < 2; z++) {
                                const float dh = z ? bf16hi(dhw[j]) : bf16lo(dhw[j]);
                                float da;
                                const float ag = activate<true>(e.act, g[2 * j + z], da);
                                const bool live = row && n + 2 * j + z < e.N;
                                dg[z] = live ? dh * u[2 * j + z] * da : 0.0f;
                                du[z] = live ? dh * ag : 0.0f;
                                hv[z] = ag * u[2 * j + z];
                            }
                            hw[j] = pack2_bf16(hv[0], hv[1]);
                            gt[j] = pack2_bf16(dg[0], dg[1]);
                            ut[j] = pack2_bf16(du[0], du[1]);
                            // a scale that is no number belongs to the columns below N alone
                            gs[j] = n + 2 * j < e.N ? pack2_bf16(dg[0] * sp, n + 2 * j + 1 < e.N ? dg[1] * sp : 0.0f) : 0u;
                            us[j] = n + 2 * j < e.N ? pack2_bf16(du[0] * sp2, n + 2 * j + 1 < e.N ? du[1] * sp2 : 0.0f) : 0u;
                        }
                        if (e.dgu) {
                            out_bf16(bx, gs, e.fp, &P.o2, nullptr, 0, n, tw, e.fp, e.T);
                            out_bf16(bx, us, e.fp, &P.o3, nullptr, 0, n, tw, e.fp, e.T);
                        }
                        if (e.dgu_t) {
                            // two neighbouring tokens of a column in one word: lanes exchange halves
                            const int64_t t2 = tw + (lane & ~1);
                            const bool in = t2 < e.ldt;
                            uint16_t* at = e.dgu_t + (n + (lane & 1)) * e.ldt + t2;
#pragma unroll
                            for (int j = 0; j < 16; j++) {
                                const uint32_t pg = __shfl_xor_sync(0xFFFFFFFFu, gt[j], 1), pu = __shfl_xor_sync(0xFFFFFFFFu, ut[j], 1);
                                const uint32_t wg = lane & 1 ? __byte_perm(pg, gt[j], 0x7632) : __byte_perm(gt[j], pg, 0x5410);
                                const uint32_t wu = lane & 1 ? __byte_perm(pu, ut[j], 0x7632) : __byte_perm(ut[j], pu, 0x5410);
                                if (in) {
                                    *reinterpret_cast<uint32_t*>(at + 2 * j * e.ldt) = wg;
                                    *reinterpret_cast<uint32_t*>(at + (e.fp + 2 * j) * e.ldt) = wu;
                                }
                            }
                        }
                    }
                    if (e.out) out_bf16(bx, hw, P.boxed, &P.o, e.out, e.ldo, n, tw, e.N, e.T);
                    if (MODE == kGated && e.h_codes) {
                        const bool live = row && n < e.N;    // N is a multiple of 32
                        uint32_t m = 0;
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            if (!live) hw[j] = 0;
                            m = max(m, max(hw[j] << 16 & 0x7FFF0000u, hw[j] & 0x7FFF0000u));
                        }
                        const uint32_t ex = m >> 23;
                        const bool finite = ex != 255;
                        bad |= !finite;
                        const uint32_t code = finite && ex > 2 ? ex - 2 : 0;
                        const float inv = __uint_as_float((254u - code) << 23);
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            u64 x[4];
#pragma unroll
                            for (int z = 0; z < 4; z++) {
                                const uint32_t two = hw[4 * j + z];
                                x[z] = finite ? pack2(bf16lo(two) * inv, bf16hi(two) * inv)
                                              : pack2(copysignf(0.0f, bf16lo(two)), copysignf(0.0f, bf16hi(two)));
                            }
                            w[j] = e2m1x8(x[0], x[1], x[2], x[3]);
                        }
                        if (live) *reinterpret_cast<uint4*>(e.h_codes + t * (e.N / 2) + n / 2) = make_uint4(w[0], w[1], w[2], w[3]);
                        sf2 |= code << (8 * c);
                    }
                }
                if (MODE == kGated && e.h_codes && (tw & ~127ll) < e.T) {    // rows of an atom that hold no token: zero
                    const int64_t n = (int64_t)tn * 128 + 64 * half;
                    *reinterpret_cast<uint16_t*>(e.h_sf + swizzle_offset(t, n >> 5, e.h_kpad4)) = (uint16_t)sf2;
                }
            }
        }
        if (lane == 0) tma_store_wait();
        if (bad && e.status) atomicOr(e.status, 1);
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && s_abort && P.e.status) atomicOr(P.e.status, kStatusTimeout);
    cluster_barrier();                                       // the other CTA signals this one's barriers no more
    if (warp == kEpiWarps + 1)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// Boxes of 64 bytes by 32 rows of a result.
bool make_box_map(CUtensorMap* m, void* ptr, bool f32, int64_t rows, int64_t cols, int64_t ld) {
    const EncodeTiledFn enc = encode_fn();
    const int es = f32 ? 4 : 2;
    if (!enc || (reinterpret_cast<uintptr_t>(ptr) & 15) || (ld * es & 15)) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(ld * es)};
    const cuuint32_t box[2] = {(cuuint32_t)(64 / es), 32};
    const cuuint32_t one[2] = {1, 1};
    return enc(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, ptr, dims, strides, box, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int KIND, int MODE>
cudaError_t launch_pair_as(const Product& p, int sms, cudaStream_t s) {
    using C = Pair<KIND>;
    PairParams P = {};
    const bool ok = make_operand_map(&P.p, p.p, KIND, p.k, 128) && make_operand_map(&P.q, p.q, KIND, p.k, 128) &&
                    (MODE == kPlain || make_operand_map(&P.p2, p.p2, KIND, p.k, 128)) &&
                    (KIND == kBf16 || (make_scale_map(&P.sp, p.p, KIND, p.k) && make_scale_map(&P.sq, p.q, KIND, p.k) &&
                                       (MODE == kPlain || make_scale_map(&P.sp2, p.p2, KIND, p.k))));
    if (!ok) return cudaErrorNotSupported;
    P.k = p.k;
    P.e = make_epilogue(p);
    // A store's box is cut at the matrix's edge in whole 16 bytes, so a box that holds a
    // ragged edge goes out by elements.
    if (p.out && make_box_map(&P.o, p.out, p.out_f32, p.q.rows, p.p.rows, p.ldo)) {
        const int64_t es = p.out_f32 ? 4 : 2;
        P.boxed = p.p.rows * es % 16 == 0 ? p.p.rows : p.p.rows / (64 / es) * (64 / es);
    }
    if (p.dgu && (!make_box_map(&P.o2, p.dgu, false, p.q.rows, p.fp, 2 * p.fp) ||
                  !make_box_map(&P.o3, static_cast<uint16_t*>(p.dgu) + p.fp, false, p.q.rows, p.fp, 2 * p.fp)))
        return cudaErrorNotSupported;
    const int64_t width = MODE == kPlain ? 256 : 128;
    P.tiles_t = (int)((p.q.rows + 255) / 256);
    P.tiles_n = (int)((p.p.rows + width - 1) / width);
    const int64_t tiles = (int64_t)P.tiles_t * P.tiles_n;
    if (tiles >= 1ll << 30) return cudaErrorNotSupported;
    const auto kernel = pair_kernel<KIND, MODE>;
    static std::atomic<bool> attr_set[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    const int64_t pairs = tiles < sms / 2 ? tiles : sms / 2;
    return launch_dependent_smem(kernel, 2 * pairs, kThreadsPair, C::kSmem, s, P);
}

template <int KIND>
cudaError_t launch_pair_mode(const Product& p, int sms, cudaStream_t s) {
    switch (p.mode) {
        case kPlain: return launch_pair_as<KIND, kPlain>(p, sms, s);
        case kGated: return launch_pair_as<KIND, kGated>(p, sms, s);
        default: return launch_pair_as<KIND, kGatedGrad>(p, sms, s);
    }
}

}  // namespace
}  // namespace mm

cudaError_t launch_pair(const Product& p, int sms, cudaStream_t s) {
    switch (p.kind) {
        case kNvfp4: return mm::launch_pair_mode<kNvfp4>(p, sms, s);
        case kMxfp4: return mm::launch_pair_mode<kMxfp4>(p, sms, s);
        default: return mm::launch_pair_as<kBf16, kPlain>(p, sms, s);
    }
}

}  // namespace nvfp4

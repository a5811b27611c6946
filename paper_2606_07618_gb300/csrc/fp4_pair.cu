// Products of many tokens, and the bf16 ones of gradients: a pair of CTAs (cta_group::2) forms
// 256 tokens by 256, 224 or 128 columns (gated: 128 gate and the same 128 up columns) and walks
// several such tiles.
//
//   out[t][n] = epilogue( sum_k q[t][k] p[n][k] )
//
// Tokens are the MMA's M side, so a thread's accumulator columns are consecutive columns of
// one row: whole sectors to store, and a block of 32 for MXFP4.  Each CTA
// loads its 128 token rows and half of the tile's columns; the leader's MMA reads both halves,
// so a stage of K costs 64 KB of loads for 256 x 256 x 128 bytes of K.  An MMA takes 128 cycles for
// 32 bytes of K of any type, a stage at least 512.  4-bit products take 606 cycles a stage in NVFP4 and 570
// in MXFP4 (8192 x 4096 x 14336 in short loops: 129 and 122 us, 7.5 and 7.9 PFLOP/s), which is what
// shared memory needs for 38 KB in and 38 out (operands and scales) at 128 bytes a cycle, 601 and 555; the
// loads alone take 530, so what L2 delivers is not far behind.  bf16: 515, MMAs.
//
// bf16 operands come as they lie: K along the rows (dg and du for d_x), or down the rows (values of
// weights and activations; dg, du for the weights' gradients), then in blocks of 64 contiguous rows by 64
// steps of K that the MMA reads along the rows.  d_x's K has two parts, gate's and up's, with a global
// scale each: an accumulator for each part, added in the epilogue.
//
//   warp 8   loads: 128 bytes of K a stage, operands and scale atoms, by TMA; completion is
//            counted on the leader's barrier
//   warp 9   (leader) copies the scale atoms of both CTAs to tensor memory and issues the MMAs
//   warps 0-7  accumulators to results, beside the next tile's MMAs
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

constexpr int kThreadsPair = (kEpiWarps + 2) * 32;

struct PairParams {
    CUtensorMap p, p2, q, sp, sp2, sq;
    int64_t k;
    int tiles_t, tiles_n, split, starve;
    int stages, stage, box;                                  // the ring: slots, bytes of one; bytes of a warp's box
    int along, part;                                         // bf16: q's rows are contiguous; stages of K's first part, or 0
    int width;                                               // columns of a tile (gated: 256, half of them gate's)
    int wide_out, wide_dh, wide_codes;                       // bytes that rows of D or h, dh, codes are aligned to: 32, 16 or fewer
    Epilogue e;
};

template <int KIND>
struct Pair {
    static constexpr int kOp = 128 * kRow;                   // a CTA's part of an operand: 16 KB
    static constexpr int kS = atoms(KIND) * kAtom;
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
__device__ __forceinline__ void commit_pair(uint32_t bar, uint32_t leader) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)(3u << leader)) : "memory");
}
// Arrival at another CTA's barrier.  What it says is about tensor memory, ordered by the
// tcgen05 fence before it; a release at cluster scope would wait for this thread's stores to
// global memory too (1300 to 2400 cycles a tile, in which the next one's MMAs stood still).
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// Tile number -> token and column tile.  Eight token tiles are walked for each column tile, so
// that the tiles in flight at one time cover a near-square of the result.
__device__ __forceinline__ void tile_at(int i, int tiles_t, int tiles_n, int& tt, int& tn) {
    const int per = 8 * tiles_n, g = i / per, first = 8 * g, rows = min(8, tiles_t - first), j = i - g * per;
    tt = first + j % rows;
    tn = j / rows;
}

__device__ __forceinline__ void st32(void* p, uint4 a, uint4 b) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w) : "memory");
}
__device__ __forceinline__ uint4 word4(const uint32_t* w) { return make_uint4(w[0], w[1], w[2], w[3]); }

__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

__device__ __forceinline__ void st_shared16(uint32_t at, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
template <int ES>
__device__ __forceinline__ uint32_t ld_shared(uint32_t at) {
    uint32_t v;
    if (ES == 4) {
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    } else {
        uint16_t h;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at) : "memory");
        v = h;
    }
    return v;
}

// W words (64 or 128 bytes) of this lane's row t0 + lane, columns n.. of a result with N columns
// and T rows.  Rows aligned to 32 bytes go out as whole sectors, a lane's own (no staging:
// TMA stores of boxes waited behind the loads in the SM's TMA queue, 7.2 us a tile of K = 4096 where
// this takes 5.9).  Other rows, and a ragged last chunk, pass through the warp's 4 KB of
// shared memory and go out by elements, a row's consecutive ones to consecutive lanes.
// WHOLE: rows aligned to 32 bytes and no ragged chunk, whatever the sizes.
template <int ES, int W, bool WHOLE = false>
__device__ __forceinline__ void put_row(const uint32_t (&w)[W], int wide, uint32_t box, void* out, int64_t ld, int64_t n,
                                        int64_t t0, int64_t N, int64_t T) {
    const int lane = threadIdx.x & 31;
    if (n >= N || t0 >= T) return;                           // the same for the warp
    if (WHOLE || (wide >= 16 && n + W * 4 / ES <= N)) {
        if (t0 + lane >= T) return;
        char* at = static_cast<char*>(out) + ((t0 + lane) * ld + n) * ES;
#pragma unroll
        for (int i = 0; i < W; i += 8) {
            if (WHOLE || wide == 32) {
                st32(at + 4 * i, word4(w + i), word4(w + i + 4));
            } else {
                *reinterpret_cast<uint4*>(at + 4 * i) = word4(w + i);
                *reinterpret_cast<uint4*>(at + 4 * i + 16) = word4(w + i + 4);
            }
        }
        return;
    }
    // 32 rows of 4 W bytes, their 16-byte parts swapped against conflicts; a row's 32 elements
    // go to the 32 lanes
    static_assert(W * 4 == 32 * ES, "32 columns");
    constexpr int kRowBytes = 4 * W, kMask = kRowBytes == 64 ? 3 : 7, kShift = kRowBytes == 64 ? 1 : 0;
    __syncwarp();
#pragma unroll
    for (int c = 0; c < W / 4; c++) st_shared16(box + lane * kRowBytes + ((c ^ (lane >> kShift & kMask)) << 4), word4(w + 4 * c));
    __syncwarp();
    const int rows = (int)(T - t0 < 32 ? T - t0 : 32);
    uint32_t v[32];                                          // all read before the first is stored
#pragma unroll
    for (int r = 0; r < 32; r++)
        v[r] = ld_shared<ES>(box + r * kRowBytes + (((lane * ES >> 4) ^ (r >> kShift & kMask)) << 4) + (lane * ES & 15));
    char* at = static_cast<char*>(out) + (t0 * ld + n + lane) * ES;
    if (n + lane < N)
#pragma unroll
        for (int r = 0; r < 32; r++, at += ld * ES) {
            if (r >= rows) continue;
            if (ES == 4)
                *reinterpret_cast<uint32_t*>(at) = v[r];
            else
                *reinterpret_cast<uint16_t*>(at) = (uint16_t)v[r];
        }
}

// What a warp makes of 32 columns n.. of its rows: lane's row t = tw + lane, tw the warp's first.
enum { kFirst = 0, kSecond = 1, kAlone = 2 };                // of a run of 64 columns, or 32 alone
struct Rows {
    const Epilogue& e;
    const PairParams& P;
    uint32_t box;                                            // the warp's box in shared memory
    float sp, sp2, sq;
    int lane;
    int64_t tw, t;
    bool bad;
    uint32_t codes0[4], code0;                               // MXFP4 form of h: a run's first 32 columns

    __device__ __forceinline__ void plain(const float (&v)[32], int64_t n) const {
        // a warp's 32 rows are of one matrix: row2 is a multiple of 128
        const bool other = e.out2 && tw >= e.row2;
        void* out = other ? e.out2 : e.out;
        const int64_t t0 = other ? tw - e.row2 : tw;
        if (e.out_f32) {
            uint32_t w[32];
#pragma unroll
            for (int j = 0; j < 32; j++) w[j] = __float_as_uint(v[j] * sp * sq);
            put_row<4, 32>(w, P.wide_out, box, out, e.ldo, n, t0, e.N, e.rows1);
        } else {
            uint32_t w[16];
#pragma unroll
            for (int j = 0; j < 16; j++) w[j] = pack2_bf16(v[2 * j] * sp * sq, v[2 * j + 1] * sp * sq);
            put_row<2, 16>(w, P.wide_out, box, out, e.ldo, n, t0, e.N, e.rows1);
        }
    }

    // dh, zero where there is no token or no column
    __device__ __forceinline__ void load_dh(uint32_t (&d)[16], int64_t n) const {
        const bool row = t < e.T;
        const uint16_t* at = e.dh + t * e.lddh + n;
        if (row && n + 32 <= e.N && P.wide_dh >= 16) {
            uint4 v[4];
            if (P.wide_dh == 32) {
                ld_stream32<false>(at, v[0], v[1]);
                ld_stream32<false>(at + 16, v[2], v[3]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) v[j] = ld_stream16<false>(at + 8 * j);
            }
#pragma unroll
            for (int j = 0; j < 4; j++) d[4 * j] = v[j].x, d[4 * j + 1] = v[j].y, d[4 * j + 2] = v[j].z, d[4 * j + 3] = v[j].w;
        } else {
#pragma unroll
            for (int j = 0; j < 16; j++) {
                const uint32_t lo = row && n + 2 * j < e.N ? at[2 * j] : 0, hi = row && n + 2 * j + 1 < e.N ? at[2 * j + 1] : 0;
                d[j] = lo | hi << 16;
            }
        }
    }

    // g and u are used up; PART: kFirst or kSecond, or kAlone
    template <int KIND, int MODE, int PART>
    __device__ __forceinline__ void gated(float (&g)[32], float (&u)[32], const uint32_t (&dhw)[16], int64_t n) {
#pragma unroll
        for (int j = 0; j < 32; j++) {
            g[j] = g[j] * sp * sq;
            u[j] = u[j] * sp2 * sq;
        }
        uint32_t hw[16];
        if (MODE == kGated) {
            activate32<false>(e.act, g, nullptr);
#pragma unroll
            for (int j = 0; j < 16; j++) hw[j] = pack2_bf16(g[2 * j] * u[2 * j], g[2 * j + 1] * u[2 * j + 1]);
        } else {
            // dh is zero where there is no token or no column, and with it dg and du.  They are rounded to bf16, by up
            // to 2^-8 each, as the operands of the products that follow: the gradients are then 0.0023 off (relative,
            // of a training step of 4096 tokens), 0.0017 of it the rounding of their own bf16.  fp16 has no room for
            // gradients' exponents nor for E8M0's; two bf16 terms would double products that are three quarters of
            // the step.
            float da[32];
            activate32<true>(e.act, g, da);
            uint32_t gt[16], ut[16];
#pragma unroll
            for (int j = 0; j < 16; j++) {
                const float d0 = bf16lo(dhw[j]), d1 = bf16hi(dhw[j]);
                hw[j] = pack2_bf16(g[2 * j] * u[2 * j], g[2 * j + 1] * u[2 * j + 1]);
                g[2 * j] *= d0;
                g[2 * j + 1] *= d1;
                ut[j] = pack2_bf16(g[2 * j], g[2 * j + 1]);
                da[2 * j] *= d0 * u[2 * j];
                da[2 * j + 1] *= d1 * u[2 * j + 1];
                gt[j] = pack2_bf16(da[2 * j], da[2 * j + 1]);
            }
            put_row<2, 16, true>(gt, 32, box, e.dgu, 2 * e.fp, n, tw, e.fp, e.T);
            put_row<2, 16, true>(ut, 32, box, e.dgu + e.fp, 2 * e.fp, n, tw, e.fp, e.T);
        }
        if (e.out) put_row<2, 16>(hw, P.wide_out, box, e.out, e.ldo, n, tw, e.N, e.T);
        if (MODE == kGated && e.h_codes) {
            const bool live = t < e.T && n < e.N;    // N is a multiple of 32
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
                    const uint32_t two = finite ? hw[4 * j + z] : hw[4 * j + z] & 0x80008000u;
                    x[z] = pack2(bf16lo(two) * inv, bf16hi(two) * inv);
                }
                w[j] = e2m1x8(x[0], x[1], x[2], x[3]);
            }
            uint8_t* at = e.h_codes + t * (e.N / 2) + n / 2;
            const bool row = (tw & ~127ll) < e.T;                // rows of an atom that hold no token: zero
            uint8_t* sf = e.h_sf + swizzle_offset(t, n >> 5, e.h_kpad4);
            if (PART == kAlone || P.wide_codes != 32) {
                if (live) *reinterpret_cast<uint4*>(at) = word4(w);
            } else if (PART == kSecond && live) {                // both blocks are there: N is a multiple of 64
                st32(at - 16, word4(codes0), word4(w));
            }
            if (PART == kAlone && row) *sf = (uint8_t)code;
            if (PART == kSecond && row) *reinterpret_cast<uint16_t*>(sf - 1) = (uint16_t)(code0 | code << 8);
#pragma unroll
            for (int j = 0; j < 4; j++) codes0[j] = w[j];
            code0 = code;
        }
    }
};

template <int KIND, int MODE, bool SPLIT>
__global__ void __launch_bounds__(kThreadsPair, 1) pair_kernel(const __grid_constant__ PairParams P) {
    using C = Pair<KIND>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kPairStages + 4];
    __shared__ int s_abort;
    __shared__ uint32_t s_tmem;
    uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
    // the CTA's place in its pair, the pair's in its cluster (which splits K), the pair's stages of K
    const uint32_t crank = cluster_rank(), rank = crank & 1, pair = SPLIT ? crank >> 1 : 0, leader = crank & ~1u;
    const int split = SPLIT ? P.split : 1;
    const int all = (int)((P.k + stage_k(KIND) - 1) / stage_k(KIND));
    const int k0 = SPLIT ? (int)((int64_t)all * pair / split) : 0, nst = SPLIT ? (int)((int64_t)all * (pair + 1) / split) - k0 : all;
    const int width = MODE == kPlain ? P.width : 256, stages = P.stages, stage = P.stage;
    const int sf_at = C::kOp + width / 2 * kRow;             // a slot: tokens, columns, scales
    const int ntiles = P.tiles_t * P.tiles_n, step = (int)gridDim.x / (2 * split), first = (int)blockIdx.x / (2 * split);
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kPairStages, accf0 = empty0 + 8 * kPairStages,
                   drained0 = accf0 + 16;

    if (tid == 0) {
        for (int b = 0; b < stages; b++) {
            mbar_init(full0 + 8 * b, 1 + P.starve);
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
        Ring ring(smem_u32(base));
        const uint32_t leader_full = at_rank(full0, leader);
        bool ok = true;
        int issued = 0;
        uint32_t swap = 0;                                   // gated: gate and up change places with the accumulators
        for (int i = first; ok && i < ntiles; i += step, swap ^= 1) {
            int tt, tn;
            tile_at(i, P.tiles_t, P.tiles_n, tt, tn);
            const int t0 = tt * 256 + (int)rank * 128;
            for (int kc = 0; kc < nst; kc++) {
                const int r = ring.slot;
                if (issued >= stages && !mbar_wait_warp(empty0 + 8 * r, ring.parity ^ 1)) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    const uint32_t st = ring.at, bar = leader_full + 8 * r;
                    if (rank == 0) mbar_expect_tx(full0 + 8 * r, 2 * stage);
                    const int x = (k0 + kc) * (KIND == kBf16 ? 64 : 128);
                    const int n = tn * width + (int)rank * (width / 2);
                    if (KIND == kBf16 && P.along) {          // 64 rows by 64 steps of K, twice
                        tma_load_2d_pair(st, &P.q, t0, x, bar);
                        tma_load_2d_pair(st + kBlock, &P.q, t0 + 64, x, bar);
                    } else {
                        tma_load_2d_pair(st, &P.q, x, t0, bar);
                    }
                    if (KIND == kBf16) {
                        tma_load_2d_pair(st + C::kOp, &P.p, n, x, bar);
                        if (width > 128) tma_load_2d_pair(st + C::kOp + kBlock, &P.p, n + 64, x, bar);
                    } else if (MODE == kPlain)
                        tma_load_2d_pair(st + C::kOp, &P.p, x, n, bar);
                    else
                        tma_load_2d_pair(st + C::kOp, rank == swap ? &P.p : &P.p2, x, tn * 128, bar);
                    if (KIND != kBf16) {
                        const uint32_t sf = st + sf_at;
                        const int a = (k0 + kc) * atoms(KIND);
                        tma_load_3d_pair(sf, &P.sq, 0, a, t0 >> 7, bar);
                        if (MODE == kPlain) {
                            tma_load_3d_pair(sf + C::kS, &P.sp, 0, a, tn * (width >> 7), bar);   // one or two atom rows
                        } else {
                            tma_load_3d_pair(sf + C::kS, swap ? &P.sp2 : &P.sp, 0, a, tn, bar);
                            tma_load_3d_pair(sf + 2 * C::kS, swap ? &P.sp : &P.sp2, 0, a, tn, bar);
                        }
                    }
                }
                __syncwarp();
                if (issued < stages) issued++;
                ring.next(stages, stage);
            }
        }
        // Every slot in use read, hence landed.  After a timeout the leader, whose barriers count both
        // CTAs' copies, waits for those instead (the other CTA stays for the last cluster barrier).
        if (issued < stages) ring = Ring(ring.first, 1);          // each used once
        const bool landed = !ok;
        if (!landed || rank == 0)
            for (int j = 0; j < issued; j++, ring.next(stages, stage))
                if (!mbar_wait_warp((landed ? full0 : empty0) + 8 * ring.slot, ring.parity ^ 1)) {
                    ok = false;
                    break;
                }
        if (!ok && lane == 0) atomicOr(&s_abort, 1);
    } else if (warp == kEpiWarps + 1 && rank == 0) {
        const uint32_t id = idesc(KIND, 256, width) | (KIND == kBf16 ? kAlongB | (P.along ? kAlongA : 0u) : 0u);
        const int second = KIND == kBf16 && P.part ? P.part - k0 : 1 << 30;    // the first stage of K's second part
        Ring ring(smem_u32(base));
        int it = 0;
        bool ok = true;
        for (int i = first; ok && i < ntiles; i += step, it++) {
            if (it > 0 && !mbar_wait_warp(drained0 + 8 * ((it - 1) & 1), ((it - 1) >> 1) & 1)) ok = false;
            tc_fence_after();
            const uint32_t acc0 = KIND == kBf16 && P.part ? tmem : tmem + (it & 1) * C::kAcc1;
            for (int kc = 0; ok && kc < nst; kc++) {
                const int r = ring.slot;
                if (!mbar_wait_warp(full0 + 8 * r, ring.parity)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                if (elect_one()) {
                    const uint32_t st = ring.at, sf = st + sf_at;
#pragma unroll
                    for (int a = 0; a < atoms(KIND); a++) {
                        cp_atom<2>(tmem + C::kSf + 4 * a, atom_desc(sf + a * kAtom));
                        cp_atom<2>(tmem + C::kSf + 16 + 8 * a, atom_desc(sf + C::kS + a * kAtom));
                        if (width > 128) cp_atom<2>(tmem + C::kSf + 16 + 8 * a + 4, atom_desc(sf + 2 * C::kS + a * kAtom));
                    }
                    const int left = (int)((P.k - (int64_t)(k0 + kc) * stage_k(KIND) + mma_k(KIND) - 1) / mma_k(KIND));
#pragma unroll
                    for (int kk = 0; kk < 4; kk++) {
                        if (kk >= left) break;
                        const int a = KIND == kNvfp4 ? kk : kk >> 1;
                        if (KIND == kBf16) {
                            // contiguous rows: 16 steps of K are 16 rows of 128 bytes, 64 rows a block
                            const uint64_t ad = P.along ? smem_desc(st + kk * 16 * kRow, kBlock, 1024) : smem_desc(st + kk * 32, 16, 1024);
                            mma<KIND, 2>(kc >= second ? acc0 + 256 : acc0, ad, smem_desc(st + C::kOp + kk * 16 * kRow, kBlock, 1024), id,
                                         (uint32_t)((kc != 0 && kc != second) | kk), 0, 0);
                        } else {
                            mma<KIND, 2>(acc0, smem_desc(st + kk * 32, 16, 1024), smem_desc(st + C::kOp + kk * 32, 16, 1024),
                                         KIND == kMxfp4 ? id | sf_id(2 * (kk & 1)) : id, (uint32_t)(kc | kk), tmem + C::kSf + 4 * a,
                                         tmem + C::kSf + 16 + 8 * a);
                        }
                    }
                    commit_pair(empty0 + 8 * r, leader);
                    if (kc == nst - 1) commit_pair(accf0 + 8 * (it & 1), leader);
                }
                __syncwarp();
                ring.next(stages, stage);
            }
        }
        if (!ok && lane == 0) atomicOr(&s_abort, 1);
    } else if (warp < kEpiWarps) {
        const Epilogue& e = P.e;
        const int half = warp >> 2, q = warp & 3;
        Rows rows{e, P, smem_u32(base) + (uint32_t)(stages * stage + warp * P.box), scale_or_1(e.s_p), scale_or_1(e.s_p2),
                  scale_or_1(e.s_q), lane};
        rows.bad = false;
        bool lost = false;                                   // a wait ran out
        // two parts of K, an accumulator and a scale each: added here, 32 columns at a time
        const bool parts = KIND == kBf16 && P.part;
        const float part0 = rows.sp, part1 = rows.sp2;
        if (parts) rows.sp = 1.0f;
        auto add_parts = [&](uint32_t at, float (&v)[32]) {
            float w[32];
            const bool a = !SPLIT || k0 < P.part, b = !SPLIT || k0 + nst > P.part;   // those this pair has
            if (a) tmem_ld32(at, v);
            if (b) tmem_ld32(at + 256, w);
            if (a) tmem_wait32(v);
            if (b) tmem_wait32(w);
#pragma unroll
            for (int j = 0; j < 32; j++) v[j] = (a ? v[j] * part0 : 0.0f) + (b ? w[j] * part1 : 0.0f);
        };
        const uint32_t leader_drained = at_rank(drained0, leader);
        int it = 0;
        for (int i = first; i < ntiles; i += step, it++) {
            int tt, tn;
            tile_at(i, P.tiles_t, P.tiles_n, tt, tn);
            rows.tw = (int64_t)tt * 256 + rank * 128 + 32 * q;
            rows.t = rows.tw + lane;
            const int b = it & 1;
            const bool overlap = KIND != kBf16 && width == 256 && half == 1 - b;   // this warp reads the overlapping columns
            auto release = [&]() {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at(leader_drained + 8 * b);
            };
            if (!overlap && !parts) release();               // done with the tile before
            uint32_t dhw[2][16];
            const int64_t n0 = MODE == kPlain ? (int64_t)tn * width : (int64_t)tn * 128 + 64 * half;
            if (MODE == kGatedGrad && !SPLIT) {              // asked for before the accumulators are waited for
                rows.load_dh(dhw[0], n0);
                rows.load_dh(dhw[1], n0 + 32);
            }
            if (!mbar_wait_warp(accf0 + 8 * b, (it >> 1) & 1)) {
                if (lane == 0) atomicOr(&s_abort, 1);
                lost = true;
                break;
            }
            tc_fence_after();
            const uint32_t acc = tmem + (parts ? 0 : b * C::kAcc1) + ((uint32_t)(32 * q) << 16);
            if (SPLIT) {                                     // sums to shared memory, in the ring's place: all its stages are read
                float* red = reinterpret_cast<float*>(base) + 32 * q + lane;
#pragma unroll 1
                for (int c = 0; c < 128 && 128 * half + c < width; c += 32) {
                    float v[32];
                    if (parts) {
                        add_parts(acc + 128 * half + c, v);
                    } else {
                        tmem_ld32(acc + 128 * half + c, v);
                        tmem_wait32(v);
                    }
#pragma unroll
                    for (int j = 0; j < 32; j++) red[(128 * half + c + j) * 128] = v[j];
                }
            } else if (MODE == kPlain && KIND == kBf16 && parts) {
                const int mid = (width + 32) / 64 * 32, end = half == 0 ? mid : width;
#pragma unroll 1
                for (int col = mid * half; col < end; col += 32) {
                    float v[32];
                    add_parts(acc + col, v);
                    if (col + 32 >= end) release();          // both accumulators are this tile's
                    rows.plain(v, n0 + col);
                }
            } else if (MODE == kPlain) {
                // the columns of this half of the warps, 64 at a time, the overlapping ones first
                const int mid = (width + 32) / 64 * 32, end = half == 0 ? mid : width;
#pragma unroll 1
                for (int c = 0; c < 2; c++) {
                    const int col = mid * half + 64 * (overlap && half == 1 ? 1 - c : c);
                    if (col >= end) break;
                    float v[2][32];
                    tmem_ld32(acc + col, v[0]);
                    tmem_ld32(acc + col + 32, v[1]);
                    tmem_wait32(v[0]);
                    tmem_wait32(v[1]);
                    if (overlap && c == 0) release();
                    rows.plain(v[0], n0 + col);
                    if (col + 32 < end) rows.plain(v[1], n0 + col + 32);
                }
            } else {
                // The up columns (the overlapping ones are theirs in either accumulator) to registers, then 32
                // gate columns at a time.
                const uint32_t up = acc + (b == 0 ? 128 : 0) + 64 * half, gate = acc + (b == 0 ? 0 : 128) + 64 * half;
                float u[2][32];
                tmem_ld32(up, u[0]);
                tmem_ld32(up + 32, u[1]);
                tmem_wait32(u[0]);
                tmem_wait32(u[1]);
                if (overlap) release();
                float g[32];
                if (MODE == kGated) {
                    tmem_ld32(gate, g);
                    tmem_wait32(g);
                    rows.gated<KIND, MODE, kFirst>(g, u[0], dhw[0], n0);
                    tmem_ld32(gate + 32, g);
                    tmem_wait32(g);
                    rows.gated<KIND, MODE, kSecond>(g, u[1], dhw[1], n0 + 32);
                } else {
                    // rolled, for the instruction cache (two copies: 311 us where this takes 223)
#pragma unroll 1
                    for (int c = 0; c < 2; c++) {
                        tmem_ld32(gate + 32 * c, g);
                        tmem_wait32(g);
                        rows.gated<KIND, MODE, kAlone>(g, u[0], dhw[0], n0 + 32 * c);
#pragma unroll
                        for (int j = 0; j < 32; j++) u[0][j] = u[1][j];
#pragma unroll
                        for (int j = 0; j < 16; j++) dhw[0][j] = dhw[1][j];
                    }
                }
            }
        }
        if (SPLIT) {
            // one tile to a cluster: each pair finishes its share of the columns, adding all
            // pairs' sums in their order; none does after a timeout anywhere in the cluster
            if (lost && lane < 2 * split) st_cluster(at_rank(smem_u32(&s_abort), lane), 1);
            __syncwarp();
            cluster_barrier();
            const bool whole = *reinterpret_cast<volatile int*>(&s_abort) == 0;
            int tt, tn;
            tile_at(first, P.tiles_t, P.tiles_n, tt, tn);
            const uint32_t mine = smem_u32(base) + 4 * (32 * q + lane);
            auto sum32 = [&](int col, float (&v)[32]) {
#pragma unroll
                for (int j = 0; j < 32; j++) v[j] = 0.0f;
                for (int r = 0; r < split; r++) {
                    const uint32_t at = at_rank(mine + col * 512, 2 * r + rank);
#pragma unroll
                    for (int j = 0; j < 32; j++) v[j] += ld_cluster(at + 512 * j);
                }
            };
            const int share = (MODE == kPlain ? width : 128) / split, from = share * (int)pair + (half * share / 2 & ~31);
            const int to = half == 0 ? share * (int)pair + (share / 2 < 32 ? 32 : share / 2) : share * (int)(pair + 1);
            if (whole && (half == 0 || share >= 64))
#pragma unroll 1
                for (int c = from; c < to; c += 32) {
                    float g[32], u[32];
                    sum32(c, g);
                    if (MODE == kPlain) {
                        rows.plain(g, (int64_t)tn * width + c);
                    } else {
                        uint32_t dhw[16];
                        const int64_t n = (int64_t)tn * 128 + c;
                        if (MODE == kGatedGrad) rows.load_dh(dhw, n);
                        sum32(128 + c, u);
                        rows.gated<KIND, MODE, kAlone>(g, u, dhw, n);
                    }
                }
        }
        if (rows.bad && e.status) atomicOr(e.status, 1);
    }
    if (SPLIT && warp >= kEpiWarps) {
        __syncwarp();
        cluster_barrier();
    }
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && s_abort && P.e.status) atomicOr(P.e.status, kStatusTimeout);
    cluster_barrier();                                       // the other CTA signals this one's barriers no more
    if (warp == kEpiWarps + 1)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// What a matrix's rows are aligned to: 32, 16 or fewer bytes (1).
int row_alignment(const void* p, int64_t stride_bytes) {
    const uintptr_t bits = reinterpret_cast<uintptr_t>(p) | (uintptr_t)stride_bytes;
    return bits % 32 == 0 ? 32 : bits % 16 == 0 ? 16 : 1;
}

template <int KIND, int MODE, bool SPLIT>
cudaError_t launch_pair_as(const Product& p, int width, int split, int sms, cudaStream_t s) {
    using C = Pair<KIND>;
    PairParams P = {};
    P.width = width;
    const int64_t tiles_t = (p.q.rows + 255) / 256;
    const bool ok = make_operand_map(&P.p, p.p, KIND, p.k, MODE == kPlain ? P.width / 2 : 128) && make_operand_map(&P.q, p.q, KIND, p.k, 128) &&
                    (MODE == kPlain || make_operand_map(&P.p2, p.p2, KIND, p.k, 128)) &&
                    (KIND == kBf16 || (make_scale_map(&P.sp, p.p, KIND, p.k, MODE == kPlain && width > 128 ? 2 : 1) && make_scale_map(&P.sq, p.q, KIND, p.k) &&
                                       (MODE == kPlain || make_scale_map(&P.sp2, p.p2, KIND, p.k))));
    if (!ok) return cudaErrorNotSupported;
    P.k = p.k;
    P.along = p.q.along;
    P.part = (int)(p.k_part / stage_k(KIND));
    P.e = make_epilogue(p);
    P.wide_out = row_alignment(p.out, p.ldo * (p.out_f32 ? 4 : 2));
    if (p.out2 && row_alignment(p.out2, 0) < P.wide_out) P.wide_out = row_alignment(p.out2, 0);
    P.wide_dh = row_alignment(p.dh, p.lddh * 2);
    P.wide_codes = row_alignment(p.h_codes, p.p.rows / 2);
    const int64_t columns = MODE == kPlain ? width : 128;
    P.tiles_t = (int)tiles_t;
    P.tiles_n = (int)((p.p.rows + columns - 1) / columns);
    const int64_t tiles = (int64_t)P.tiles_t * P.tiles_n;
    if (tiles >= 1ll << 30) return cudaErrorNotSupported;
    const auto kernel = pair_kernel<KIND, MODE, SPLIT>;
    static std::atomic<bool> attr_set[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPairSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    P.split = split;
    P.stage = stage_bytes(KIND, width);
    P.box = box_bytes(p.out_f32);
    P.stages = ring_slots(p.sizes(), width);
    P.starve = p.starve;
    const int64_t pairs = SPLIT ? tiles * split : tiles < sms / 2 ? tiles : sms / 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * pairs));
    cfg.blockDim = dim3(kThreadsPair);
    cfg.dynamicSmemBytes = (size_t)(P.stages * P.stage + kEpiWarps * P.box + 1024);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)(2 * split);
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, P);
}

template <int KIND, int MODE>
cudaError_t launch_pair_mode(const Product& p, int sms, cudaStream_t s) {
    const PairPlan b = pair_plan(p.sizes(), sms);
    return b.split > 1 ? launch_pair_as<KIND, MODE, true>(p, b.width, b.split, sms, s)
                       : launch_pair_as<KIND, MODE, false>(p, b.width, 1, sms, s);
}

template <int KIND>
cudaError_t launch_pair_kind(const Product& p, int sms, cudaStream_t s) {
    switch (p.mode) {
        case kPlain: return launch_pair_mode<KIND, kPlain>(p, sms, s);
        case kGated: return launch_pair_mode<KIND, kGated>(p, sms, s);
        default: return launch_pair_mode<KIND, kGatedGrad>(p, sms, s);
    }
}

}  // namespace
}  // namespace mm

cudaError_t launch_pair(const Product& p, int sms, cudaStream_t s) {
    switch (p.kind) {
        case kNvfp4: return mm::launch_pair_kind<kNvfp4>(p, sms, s);
        case kMxfp4: return mm::launch_pair_kind<kMxfp4>(p, sms, s);
        default: return mm::launch_pair_mode<kBf16, kPlain>(p, sms, s);
    }
}

}  // namespace nvfp4

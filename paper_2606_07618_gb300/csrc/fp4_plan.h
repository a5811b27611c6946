// How a product is cut up: which kernel forms it, how wide a tile is and how many CTAs or
// pairs share its K.  Host code without CUDA, so that the choices can be checked without a GPU.
#pragma once
#include <cstdint>
#include <initializer_list>

#ifdef __CUDACC__
#define NVFP4_BOTH __host__ __device__
#else
#define NVFP4_BOTH
#endif

namespace nvfp4 {

enum { kNvfp4 = 0, kMxfp4 = 1, kBf16 = 2 };                  // operand kinds of a product
enum { kPlain = 0, kGated = 1, kGatedGrad = 2 };             // what the epilogue makes of the accumulators

namespace mm {

// An operand tile is staged as rows of 128 bytes (one swizzle row) along K: 256 codes or
// 64 bf16, four MMAs of 32 bytes each.  Scales come as 512-byte atoms of 128 rows by
// four scale columns, 64 (NVFP4) or 128 (MXFP4) elements of K.
NVFP4_BOTH constexpr int stage_k(int kind) { return kind == kBf16 ? 64 : 256; }
NVFP4_BOTH constexpr int mma_k(int kind) { return kind == kBf16 ? 16 : 64; }
NVFP4_BOTH constexpr int atoms(int kind) { return kind == kNvfp4 ? 4 : kind == kMxfp4 ? 2 : 0; }
constexpr int kAtom = 512;
constexpr int kRow = 128;                                    // bytes of an operand row in a stage

// A product's sizes: out[t][n] from sums over k; ldq: row stride of a bf16 q in elements.
struct Sizes {
    int kind, mode, out_f32;
    int64_t t, n, k, ldq;
    int64_t stages() const { return (k + stage_k(kind) - 1) / stage_k(kind); }
};

// Up to 32 tokens the weight is streamed past them, up to 64 where it is long or has a tile for
// half the SMs; more go to pairs of CTAs.  us, here / pairs: 32 x 1024 x 1024 4.4 / 4.8, 32 x 2048 x 2048
// 4.7 / 6.0, gated 32 x 14336 x 4096 14.1 / 19.0; 64 x 4096 x 14336 12.4 / 16.7, 64 x 14336 x 4096 9.7 /
// 10.2, gated 15.7 / 18.0; 64 x 1024 x 1024 6.9 / 5.0, 64 x 4096 x 4096 9.1 / 8.3, gated 64 x 2048 x 2048
// 11.0 / 6.8.
inline bool few_tokens(const Sizes& p, int sms) {
    if (p.kind == kBf16 || p.mode == kGatedGrad) return false;
    const bool long_or_wide = p.k >= 8192 || 2 * ((p.n + 127) / 128) > sms;
    return p.t <= (long_or_wide ? 64 : 32);
}

// Few tokens: CTAs that share the K of a tile of 128 columns, and whether a CTA has a whole SM's ring.
struct TilePlan {
    int log_split;
    bool whole;
};
inline TilePlan tile_plan(const Sizes& p, int sms) {
    const int64_t tn = (p.n + 127) / 128, nst = p.stages();
    // Few tiles: up to eight CTAs to a tile, two to an SM, so that some 150 to 300 load (us with
    // 8 / 4 / 2 at most: 1 x 4096 x 4096 4.2 / 4.3 / 5.1, 1 x 4096 x 14336 7.0 / 8.6 / 11.4, gated 1 x
    // 4096 x 4096 4.9 / 5.6 / 7.3).  Past half the SMs a CTA to a tile with the whole SM's ring: gated
    // 16 x 14336 x 4096 14.7, where two with half a ring take 15.5; 64 x 14336 x 4096 11.3 / 16.6.
    TilePlan b = {0, false};
    const bool share = 2 * tn <= sms;
    while (share && b.log_split < 3 && 5 * (tn << b.log_split) < 6 * sms && (2 << b.log_split) <= nst) b.log_split++;
    b.whole = !share && tn <= sms;
    return b;
}

// Pairs of CTAs.
constexpr int kEpiWarps = 8;
constexpr int kPairStages = 8;                               // at most
constexpr int kBlock = 64 * kRow;                            // 64 contiguous rows by 64 steps of K, bf16
constexpr int kPairSmem = 227 * 1024 - 256;                  // of a CTA, less its static part

// A slot of the ring: 128 rows of tokens, half a tile's columns (bf16: in blocks of 64), their
// scales.  A multiple of 1024.
inline int stage_bytes(int kind, int width) {
    if (kind == kBf16) return (width > 128 ? 4 : 3) * kBlock;
    return (128 + width / 2) * kRow + (width > 128 ? 3 : 2) * atoms(kind) * kAtom;
}
// A warp's box: 32 x 32 elements of a result whose rows allow no wide store.
inline int box_bytes(int out_f32) { return out_f32 ? 4096 : 2048; }
inline int ring_slots(const Sizes& p, int width) {
    const int n = (kPairSmem - 1024 - kEpiWarps * box_bytes(p.out_f32)) / stage_bytes(p.kind, width);
    return n > kPairStages ? kPairStages : n;
}

// How wide a tile is and how many pairs share its K: the least of an estimate in cycles.
//   A stage takes its MMAs (2 a column) or its loads, 55 to 70 bytes a cycle and CTA with most SMs
//   loading, 100 with few, or its share of the latency of HBM; a tile 1500 more, adding up a split K
//   8000.  Narrow tiles fill the last wave (bf16 224 too; 192 and 160 load as much as that, for fewer
//   columns; a 4-bit tile takes whole scale atoms of 128 rows, so it is 256 or 128 wide and a gated one
//   256) and shorten what a few tiles take; clusters of four or eight whole SMs have to find room (at
//   most 36 and 15 on a GB300: 16 of eight ran one after the others).
// us, always 256 wide and split from 32 stages on / as estimated: 77 x 1001 x 2080 (fp32) 7.9 / 6.4, 512 x
// 1024 x 1024 6.0 / 5.1, 256 x 4096 x 14336 17.8 / 15.7, 200 x 512 x 14336 13.4 / 10.8; with gradients 2048
// x 4096 x 4096 111 / 106.
struct PairPlan {
    int width = 256, split = 1;
};
inline PairPlan pair_plan(const Sizes& p, int sms) {
    const int64_t pairs = sms > 1 ? sms / 2 : 1, tiles_t = (p.t + 255) / 256, nst = p.stages();
    // bf16 rows that start inside a 128-byte line take two of L2's
    const int64_t full_rate = p.kind != kBf16 ? 62 : p.ldq % 64 == 0 ? 70 : 55;
    PairPlan best;
    int64_t least_cost = INT64_MAX;
    for (const int w : {256, 224, 128}) {
        if (w != 256 && (p.mode != kPlain || (w == 224 && p.kind != kBf16))) continue;
        const int64_t columns = p.mode == kPlain ? w : 128, tiles = tiles_t * ((p.n + columns - 1) / columns);
        const int64_t bytes = stage_bytes(p.kind, w), latency = 2900 / ring_slots(p, w);
        for (int split = 1; split <= 4; split *= 2) {
            if (split > 1 && (w % 128 != 0 || nst < 8 * split || tiles > (split == 2 ? sms / 4 - 2 : sms / 8 - 4))) continue;
            const int64_t rate = 2 * tiles * split > pairs ? full_rate : 100;
            const int64_t moved = bytes / rate > latency ? bytes / rate : latency, stage = moved > 2 * w ? moved : 2 * w;
            const int64_t waves = split > 1 ? 1 : (tiles + pairs - 1) / pairs;
            const int64_t cost = waves * ((nst + split - 1) / split * stage + 1500) + (split > 1 ? 8000 : 0);
            if (least_cost == INT64_MAX || 32 * cost < 31 * least_cost) {   // not for a difference the estimate cannot see
                least_cost = cost;
                best.width = w;
                best.split = split;
            }
        }
    }
    return best;
}

}  // namespace mm
}  // namespace nvfp4

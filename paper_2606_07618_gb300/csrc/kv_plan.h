// How attention over the cache is cut up: plain arithmetic on the sizes that the host knows
// (no CUDA), shared by the workspace query, the launches and the tests.
#pragma once
#include <cstdint>

namespace nvfp4 {
namespace kv {

// Few rows (kv_attention.cu): a warp takes 64 tokens at a time, a block has four warps, and an SM holds as many blocks as
// their registers allow without spilling (dim 128 and 8 rows: 22.4 us in four, 26.3 in five of 96 registers).  Parts of one
// sequence and head join in a cluster of up to 8 blocks, more of them through the workspace.
constexpr int kWarpTokens = 64, kMaxCluster = 8;
constexpr int64_t kSms = 152;
constexpr int blocks_per_sm(int64_t dim, int rows) { return dim == 128 ? (rows == 8 ? 4 : 2) : (rows == 8 ? 5 : 4); }
// Many rows (kv_attention_tile.cu): rows of a block, one to an SM, and the keys that it takes at a time.
constexpr int kTileRows = 256, kTileKeys = 128, kPairRows = 512;     // (of a pair of blocks, dim 128)

// Most tokens that a table can hold: the kernels' token numbers are ints, which pass the last token by up to a block's start
// (192), two tiles of 256 and 48 within one, and a part's tokens round up to a step.
constexpr int64_t kMaxLength = ((int64_t)1 << 31) - 2048;

struct Sizes {
    int64_t tokens, batch, max_q;        // rows of q, sequences, the most queries of one
    int q_heads, heads, dim;
    int64_t length, prefix;              // the most cached tokens that the tables hold
};

#ifdef __CUDACC__
#define KV_BOTH __host__ __device__
#else
#define KV_BOTH
#endif

// One pass over keys: rows of a key head in tiles of `rows`, keys in `parts`.
struct Pass {
    int rows;
    int64_t tiles, parts;
    KV_BOTH int64_t step() const { return rows >= kTileRows ? kTileKeys : kWarpTokens; }
};

// Tokens of a part of a sequence of `length`: the parts are as even as whole steps allow.
KV_BOTH inline int64_t part_tokens(int64_t length, int64_t parts, int64_t step) {
    const int64_t n = (length + parts * step - 1) / (parts * step);
    return (n < 1 ? 1 : n) * step;
}

KV_BOTH inline uint32_t part_tokens32(uint32_t length, uint32_t parts, uint32_t step) {      // length below 2^31
    const uint32_t n = (length + parts * step - 1) / (parts * step);
    return (n < 1 ? 1 : n) * step;
}

struct Plan {
    Pass own, prefix;                    // prefix.parts is 0 without one
    int64_t parts() const { return own.parts + prefix.parts; }
    // Whether parts' sums go through the workspace: [parts][tokens][q_heads][dim] fp32, then maxima and sums of weights.  With
    // `merge` those of the prefix alone, whose pass comes first: the pass over each sequence's own keys adds them to its results.
    // Else the own parts, then the prefix's, and a launch of its own joins them.
    bool through = false, merge = false;
    int64_t values = 0, bytes = 0;
    bool small = true;
    // Whether the launches' grids can hold it.
    bool fits() const { return small; }
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Parts of a few rows' pass.  Blocks of equal work run in whole waves; of sequences between nothing and `length` tokens the
// average is half of that, and the last block to start may be a longest one.  A block costs as much as kBlockCost
// tokens before and after its loop.  The parts for which the two estimates together are least are taken, of the
// cluster sizes that fill the GPU's groups of SMs evenly (16 sequences of 4096 tokens and 8 heads: 20.6 us in 2 parts, 24.5 in
// 3, 19.8 in 4, 23.9 in 8; 37 of up to 20000 tokens, 4 heads: 68, 65, 52, 49).
inline int64_t thin_parts(int64_t pairs, int64_t length, int64_t slots) {
    constexpr int64_t kBlockCost = 384;
    if (pairs * kMaxCluster <= slots) {  // few: blocks of 128 tokens or more in a cluster, or of 256 and as many as there is room for
        const int64_t n = ceil_div(length, 2 * kWarpTokens), most = ceil_div(length, 4 * kWarpTokens), all = slots / pairs;
        if (most <= kMaxCluster) return n < 2 ? 1 : n < 4 ? 2 : n < kMaxCluster ? 4 : kMaxCluster;
        return most < all ? most : all;
    }
    int64_t best = 1, least = INT64_MAX;
    for (int64_t n = 1; n <= kMaxCluster; n *= 2) {
        if (n > 1 && (n - 1) * 2 * kWarpTokens >= length) break;
        const int64_t block = kBlockCost + length / n, waves = ceil_div(pairs * n, slots);
        const int64_t ragged = waves == 1 ? block : pairs * n * (kBlockCost + length / n / 2) / slots + block;
        if (waves * block + ragged < least) least = waves * block + ragged, best = n;
    }
    return best;
}

// Up to 16 rows of a sequence and key head go to the kernel that holds them in registers (16 rows take 1.4 times what 8 do),
// more to the tensor cores' tiles, where 17 cost what 128 do.
inline Pass plan_pass(int64_t sequences, int64_t heads, int64_t dim, int64_t rows, int64_t length) {
    Pass p;
    p.rows = rows <= 8 ? 8 : rows <= 16 ? 16 : kTileRows;
    p.tiles = ceil_div(rows, p.rows);
    p.parts = 1;
    if (length <= 0 || sequences > kSms * 64 || p.tiles > kSms * 64) return p;      // (their product would be that, too)
    const int64_t pairs = sequences * heads * p.tiles;
    if (p.rows < kTileRows) {
        p.parts = thin_parts(pairs, length, kSms * blocks_per_sm(dim, p.rows));
    } else {
        // Two blocks' MMAs together read half the keys each: a step is a tenth shorter, the start 2 us longer.  So: pairs where
        // their rows are four fifths full and their parts long (32 heads of 2 x 2048 queries over 8192 tokens 418 -> 375 us, of
        // 16 x 104 over 4096 155 -> 133; 16 of 512 over 2048 71.5 -> 70.9; 64 x 8 of 512 over 512 118 -> 149, of 1 over 8192, in
        // parts of 900, 36.2 -> 38.7).
        constexpr int64_t kPairTokens = 2048;
        const int64_t whole = ceil_div(rows, kPairRows), two = kSms / 2 / (sequences * heads * whole);
        if (dim == 128 && whole * kPairRows <= rows + rows / 4 && length >= kPairTokens * (two < 1 ? 1 : two)) {
            p.rows = kPairRows;
            p.tiles = whole;
            p.parts = two;
        } else if (pairs < kSms) {
            const int64_t most = ceil_div(length, kTileKeys);
            p.parts = kSms / pairs < most ? kSms / pairs : most;
        }
    }
    if (p.parts < 1) p.parts = 1;
    return p;
}

inline Plan make_plan(const Sizes& s) {
    const int64_t group = s.q_heads / s.heads;
    Plan p;
    p.own = plan_pass(s.batch, s.heads, s.dim, s.max_q * group, s.length);
    p.prefix = Pass{0, 0, 0};
    if (s.prefix > 0) p.prefix = plan_pass(1, s.heads, s.dim, s.tokens * group, s.prefix);
    const int64_t blocks = (int64_t)1 << 31, rows = s.tokens * s.q_heads;
    p.small = p.own.tiles < blocks / 2 / p.own.parts / s.batch && p.prefix.tiles < blocks / 2 / (p.prefix.parts + 1) && rows < blocks;
    const bool alone = p.own.rows < kTileRows && p.own.parts <= kMaxCluster;       // the own pass needs no workspace
    p.merge = s.prefix > 0 && alone;
    p.through = p.parts() > 1 && !(s.prefix <= 0 && alone);
    if (p.small && p.through) {
        const int64_t parts = p.merge ? p.prefix.parts : p.parts();
        p.values = parts * s.tokens * s.q_heads * s.dim * 4;
        p.values = (p.values + 255) / 256 * 256;
        p.bytes = p.values + (parts * s.tokens * s.q_heads * 8 + 255) / 256 * 256;
    }
    return p;
}

}  // namespace kv
}  // namespace nvfp4

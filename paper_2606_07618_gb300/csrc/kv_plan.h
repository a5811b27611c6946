// How attention over the cache is cut up: plain arithmetic on the sizes that the host knows
// (no CUDA), shared by the workspace query, the launches and the tests.
#pragma once
#include <cstdint>

namespace nvfp4 {
namespace kv {

// Tokens of the cache that one warp takes at a time, and one block.
constexpr int kWarpTokens = 64, kBlockTokens = 256;
// Blocks that fill the GPU about twice: 152 SMs with four of them each.
constexpr int64_t kBlocks = 152 * 4 * 2;
// Rows of a block on tcgen05 (one block an SM), keys that it takes at a time.
constexpr int kTileRows = 256, kTileKeys = 128;
constexpr int64_t kTileBlocks = 152;

struct Sizes {
    int64_t tokens, batch, max_q;        // rows of q, sequences, the most queries of one
    int q_heads, heads, dim;
    int64_t length, prefix;              // the most cached tokens that the tables hold
};

// One pass over keys: rows of a key head in tiles of `rows`, keys in `parts` of `chunk` tokens.
struct Pass {
    int rows;
    int64_t tiles, parts, chunk;
};

struct Plan {
    Pass own, prefix;                    // prefix.parts is 0 without one
    int64_t parts() const { return own.parts + prefix.parts; }
    // Sums of the parts, [parts][tokens][q_heads][dim] fp32, and their maxima and sums of weights.
    int64_t values = 0, bytes = 0;
    bool small = true;
    // Whether the launches' grids can hold it.
    bool fits() const { return small; }
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline Pass plan_pass(int64_t sequences, int64_t heads, int64_t rows, int64_t length) {
    Pass p;
    p.rows = rows <= 8 ? 8 : rows <= 16 ? 16 : kTileRows;
    p.tiles = ceil_div(rows, p.rows);
    const bool tile = p.rows == kTileRows;
    const int64_t step = tile ? kTileKeys : kBlockTokens;
    const int64_t most = length > step ? ceil_div(length, step) : 1;
    int64_t parts = (tile ? kTileBlocks : kBlocks) / sequences / heads / p.tiles;
    parts = parts < 1 ? 1 : parts > most ? most : parts;
    p.chunk = ceil_div(length > 0 ? length : 1, parts * step) * step;
    p.parts = length > 0 ? ceil_div(length, p.chunk) : 1;
    return p;
}

inline Plan make_plan(const Sizes& s) {
    const int64_t group = s.q_heads / s.heads;
    Plan p;
    p.own = plan_pass(s.batch, s.heads, s.max_q * group, s.length);
    p.prefix = Pass{0, 0, 0, 0};
    if (s.prefix > 0) p.prefix = plan_pass(1, s.heads, s.tokens * group, s.prefix);
    const int64_t blocks = (int64_t)1 << 31, rows = s.tokens * s.q_heads;
    p.small = p.own.tiles < blocks / p.own.parts / s.batch && p.prefix.tiles < blocks / (p.prefix.parts + 1) && rows < 8 * blocks;
    if (p.small && p.parts() > 1) {
        p.values = p.parts() * s.tokens * s.q_heads * s.dim * 4;
        p.values = (p.values + 255) / 256 * 256;
        p.bytes = p.values + (p.parts() * s.tokens * s.q_heads * 8 + 255) / 256 * 256;
    }
    return p;
}

}  // namespace kv
}  // namespace nvfp4

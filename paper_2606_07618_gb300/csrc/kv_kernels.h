// Internal interface between the host layer of nvfp4kv.h (kv_api.cu) and its kernels.
// Not part of the public ABI.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "kv_plan.h"

namespace nvfp4 {
namespace kv {

constexpr int kStatusNonFinite = 1;      // a token's x / S is not finite
constexpr int kStatusBounds = 4;         // a length, slot or page number outside its bounds

// A key's weight is 2^(x f + (7 - m)): x its score, f the factor that makes scores logits of base 2, m the row's largest logit so far, x f
// rounded; one fused operation on a rounded 7 - m.  |x| < 2 * 128 * 2688 < 2^20, so with f <= kWideFactor logits are below 2^22
// and the two roundings, the same for all of a row's weights, small.  With larger factors the weight of m's own key could be anywhere
// (from 2^-64 to 2^64 at 2^30): there scores become rounded logits first, and f is 1, so that differences of close ones are exact.
// 7 - m, and m + 8, past which a maximum is followed, are rounded down: weights stay within 2^15 however coarse fp32 is there.
// What 7 - m lost, at most 7, is taken out of a wide row's sums at the end, where parts are joined by their m.
constexpr float kWideFactor = 4.0f;

struct Cache {
    uint8_t *codes, *sf;                 // [pages][heads][2][page][dim/2], [pages][heads][2][dim/16][page]
    const float *S_k, *S_v;
    int64_t pages;
    int page_log2, heads, dim;
};

// Strided tensor [tokens, heads, dim]; vec: base and strides are multiples of 16 bytes (1) or 32 (2).
struct Tensor {
    void* p;
    int64_t token, head;
    int vec;
};

struct Rope {
    Tensor x, out;
    int dtype, heads, dim, rot, halves, inverse;
    int64_t tokens;
    const int64_t* positions;
    const uint64_t* turns;
    float magnitude;
};

struct Write {
    Cache c;
    Tensor in[2];                        // k, v; null pointers are not written
    int dtype, method;                   // method: 0 sweep, 1 block maximum
    int64_t tokens;
    const int64_t* slots;
    int* status;
};

struct Read {
    Cache c;
    Tensor out[2];
    int dtype;
    const int32_t *table, *starts, *offsets;
    int64_t table_ld, width, batch, tokens;
    int* status;
};

struct Attention {
    Cache c;
    Tensor q, out;
    int q_heads, group, causal;
    int64_t tokens, batch, max_q;
    const int32_t *table, *lens, *offsets;
    int64_t table_ld, width;
    const int32_t *prefix, *prefix_len;  // null without a prefix
    int64_t prefix_width;
    float scale;
    float* lse;
    int* status;
    void* workspace;
    Plan plan;
    // Set for the second pass of a call.  It is launched as a dependent of the first, whose blocks let it start only once
    // they have waited for what came before the call themselves; so it does not wait for the first before it merges
    // its results, or before its end (which the join then waits for).
    int second;
    int starve;                          // 1: the waits for keys run out, 2: those for values (self-test)
};

cudaError_t launch_rope(const Rope& p, int sms, cudaStream_t s);
cudaError_t launch_write(const Write& p, int sms, cudaStream_t s);
cudaError_t launch_read(const Read& p, int sms, cudaStream_t s);
cudaError_t launch_attention(const Attention& p, cudaStream_t s);
// A pass of attention for many rows (kv_attention_tile.cu).
cudaError_t launch_tiles(const Attention& p, const Pass& pass, bool prefix, int64_t part0, cudaStream_t s);

}  // namespace kv
}  // namespace nvfp4

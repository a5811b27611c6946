/*
 * nvfp4kv.h -- C ABI of libnvfp4ss.so, third part: a key/value cache in NVFP4 and what a
 * serving program does with it.  Rotary positions, tokens quantised as they are written
 * into the cache and read back, and attention over the cached tokens, also for a batch
 * whose sequences share a long prefix, on NVIDIA GB300 (sm_103a).
 *
 * The cache is a pool of pages of `page` tokens (a power of two, 16 to 1024):
 *   codes  [pages][heads][2][page][dim/2]   packed E2M1 nibbles (nvfp4ss.h): keys, then values
 *   sf     [pages][heads][2][dim/16][page]  E4M3 scale codes of blocks of 16 along dim; the
 *          tokens of a block lie side by side, which is how attention reads them
 *   S_k, S_v  the fp32 global scales of all keys and of all values, in device memory
 *          (calibrated once; S of nvfp4_global_scale).  A value is q * s * S.
 * dim is 64 or 128.  Sequence b's token j lies at offset j % page of page
 * table[b * table_ld + j / page].  Pages may be shared by several sequences.
 *
 * Conventions are those of nvfp4ss.h and nvfp4mm.h: device-accessible pointers that the
 * caller owns, no allocation and no synchronisation, every call asynchronous on `stream`
 * and good for a CUDA graph, argument errors returned before any launch.  Sizes that only the
 * device knows (lengths, offsets, page numbers) are checked there: what lies outside
 * the stated bounds is skipped, as said at each call, and sets bit 2 (4) of status_dev.
 *   - Strides are in elements; the innermost dimension is contiguous.  Tensors need their
 *     element's alignment, and run faster with bases and strides of 16 bytes.
 *   - codes and sf are 16-byte aligned.
 *   - status_dev: optional device int; bit 0 is OR-ed in where a token to be written
 *     holds a NaN or an infinity, bit 2 as above, bit 4 (16) when a bounded wait inside a
 *     kernel ran out (about a second; the outputs are then incomplete).
 *   - Outputs must not overlap inputs or each other, but where a call says so.
 *   - No result depends on timing: sums split over several thread blocks are added in a
 *     fixed order, which follows from the sizes and widths that the host gives, so the same
 *     rows in calls of other sizes may differ in the last places.
 */
#ifndef NVFP4KV_H
#define NVFP4KV_H

#include "nvfp4ss.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    uint8_t* codes;
    uint8_t* sf;
    const float* S_k;
    const float* S_v;
    int64_t pages;
    int32_t page, heads, dim;
} nvfp4_kv_cache;

/* Which elements of a head form a pair: 2i and 2i + 1, or i and i + rot/2. */
typedef enum { NVFP4_ROPE_NEIGHBOURS = 0, NVFP4_ROPE_HALVES = 1 } nvfp4_rope_layout;
typedef enum { NVFP4_KV_ABSMAX = 0, NVFP4_KV_SWEEP = 1 } nvfp4_kv_method;
typedef enum {
    NVFP4_ROPE_PLAIN = 0,
    NVFP4_ROPE_LINEAR = 1,   /* every frequency / factor */
    NVFP4_ROPE_BASE = 2,     /* base * factor^(rot/(rot-2)): the slowest / factor, the fastest as it is */
    NVFP4_ROPE_BANDS = 3     /* by turns over the original length: / factor below `slow`, kept above `fast` */
} nvfp4_rope_scaling;

/*
 * The frequency table of rotary positions, on the host: pair i turns by
 *   f_i = base^(-2i/rot) / (2 pi) a position (rot even, 2 to 1024; base > 1),
 * scaled for contexts `factor` (>= 1) times as long as the original_len tokens a model was
 * trained on: as `scaling` says, and for NVFP4_ROPE_BANDS with r = original_len * f_i and
 * g = clamp((r - slow) / (fast - slow), 0, 1),  f_i' = f_i ((1 - g) / factor + g), 0 <= slow < fast.
 *   turns  [rot/2] host memory: round(f_i' * 2^64), fractions of a turn in 64-bit fixed point.
 * original_len, slow and fast are read for NVFP4_ROPE_BANDS alone, factor not for NVFP4_ROPE_PLAIN.
 */
nvfp4_status nvfp4_rope_turns(int rot, double base, nvfp4_rope_scaling scaling, double factor, double original_len,
                              double slow, double fast, uint64_t* turns);

/*
 * Rotary positions.  For token t, every head and pair (a, b) of the first `rot` elements,
 * with the angle u = 2 pi frac(positions[t] * turns[i] / 2^64), which 64-bit arithmetic
 * modulo 2^64 gives exactly for positions of any size and sign:
 *   a' = m (a cos u - b sin u),  b' = m (a sin u + b cos u),   m = magnitude
 * in fp32, rounded once to the type; the other dim - rot elements are copied.  `inverse`
 * turns back, by -u (with the same m): the gradient with respect to x, given that of out.
 *   x, out  [tokens, heads, dim] of type dt (NVFP4_IN_BF16, NVFP4_IN_F32), strides of a token and a head; at most
 *           2^31 - 1 tokens, 65535 heads, dim even, up to 1024, rot even and at most dim.  out may be x with the same strides.
 *   positions  [tokens]; turns [rot/2] in device memory (nvfp4_rope_turns, copied there).
 * Query and key heads that lie side by side are one tensor: one call rotates both.
 */
nvfp4_status nvfp4_rope(const void* x, int64_t x_token, int64_t x_head, void* out, int64_t out_token, int64_t out_head,
                        nvfp4_dtype dt, int64_t tokens, int heads, int dim, int rot, const int64_t* positions,
                        const uint64_t* turns, float magnitude, nvfp4_rope_layout layout, int inverse, void* stream);

/*
 * New tokens into the cache: k and v [tokens, heads, dim] of type dt, each block of 16
 * quantised by the arithmetic contract of nvfp4ss.h with S_k or S_v -- its scale that of
 * absmax_quantize (NVFP4_KV_ABSMAX) or the argmin of scalesweep_quantize with the MSE
 * objective and its default window (NVFP4_KV_SWEEP): the same codes.
 *   slots  [tokens] place of each token: page number * page + offset.  A negative slot
 *          skips its token (padding); one past the pool does too and sets bit 2.  Slots of one call
 *          are distinct; where they are not, what the slot holds is not specified.
 *   k or v may be NULL: the other alone is written.
 */
nvfp4_status nvfp4_kv_write(const nvfp4_kv_cache* cache, const void* k, int64_t k_token, int64_t k_head, const void* v,
                            int64_t v_token, int64_t v_head, nvfp4_dtype dt, int64_t tokens, const int64_t* slots,
                            nvfp4_kv_method method, int* status_dev, void* stream);

/*
 * Cached tokens read back: rows offsets[b] .. offsets[b+1] of k and v [tokens, heads, dim]
 * receive tokens starts[b], starts[b] + 1, ... of sequence b, x_hat = fl32(fl32(q s) S) as fp32 or its
 * RNE bf16.
 *   table    [batch] rows of `width` page numbers, table_ld apart; starts [batch] (NULL: all 0);
 *   offsets  [batch + 1], not falling, from 0 to at most `tokens`.  Rows past offsets[batch] are left as they are; rows
 *            whose page is outside the table or the pool become 0 and set bit 2.
 *   k or v may be NULL.
 */
nvfp4_status nvfp4_kv_read(const nvfp4_kv_cache* cache, const int32_t* table, int64_t table_ld, int64_t width,
                           const int32_t* starts, const int32_t* offsets, int64_t batch, void* k, int64_t k_token,
                           int64_t k_head, void* v, int64_t v_token, int64_t v_head, nvfp4_dtype out_dt, int64_t tokens,
                           int* status_dev, void* stream);

/*
 * Attention over the cache.  Sequence b has n = offsets[b+1] - offsets[b] queries, rows
 * offsets[b].. of q, and lens[b] cached tokens, the queries' own among them (written
 * before).  Query i sees tokens j <= lens[b] - n + i (causal), or all lens[b] of them:
 *   out = sum_j softmax_j(scale q.k_j) v_j,   lse = ln sum_j exp(scale q.k_j),
 * query head h with the keys and values of head h / (q_heads / heads).  A query that sees
 * nothing gets out = 0 and lse = -inf.  Cached values and queries are exact in the products
 * (the queries up to 2^-25 of their row's largest), sums and softmax statistics in fp32; the weights are rounded to fp16
 * (by up to 2^-11, those below 2^-21 of the row's largest by up to 2^-32 of it, 2^-25 where logits pass 2^22) for the
 * product with the values, and the result once to bf16.  Logits (of base 2, scale q.k log2 e) are rounded to fp32 and may have any size
 * that it holds: a key whose logit lies far above the others' takes all the weight, keys that tie share it.
 *   q, out  [tokens, q_heads, dim] bf16, strides of a token and a head; q_heads a multiple of
 *           the cache's heads.  lse optional [tokens, q_heads] fp32.
 *   table   [batch] rows of `width` page numbers, table_ld apart; entries behind a
 *           sequence's last page are not read; width * page at most 2^31 - 2048.  lens past width * page
 *           count as that and set bit 2; a page number outside the pool hides its tokens and sets bit 2.
 *   offsets [batch + 1], not falling, from 0 to at most `tokens`; no sequence has more than max_q queries (those past
 *           it are not computed).  Rows past offsets[batch] are left as they are.
 *   scale   finite and >= 0.
 *   workspace  nvfp4_kv_attention_workspace bytes, 256-byte aligned, with prefix_width 0; its
 *           contents need no initialisation and say nothing after the call.
 */
size_t nvfp4_kv_attention_workspace(const nvfp4_kv_cache* cache, int64_t tokens, int q_heads, int64_t batch,
                                    int64_t width, int64_t max_q, int64_t prefix_width);
nvfp4_status nvfp4_kv_attention(const nvfp4_kv_cache* cache, const void* q, int64_t q_token, int64_t q_head,
                                int64_t tokens, int q_heads, const int32_t* table, int64_t table_ld, int64_t width,
                                const int32_t* lens, const int32_t* offsets, int64_t batch, int64_t max_q, float scale,
                                int causal, void* out, int64_t out_token, int64_t out_head, float* lse, int* status_dev,
                                void* workspace, size_t ws_bytes, void* stream);

/*
 * Self-test of the bounded waits (failure detection): nvfp4_kv_attention, of more than 16 rows a
 * sequence and key head (max_q * q_heads / heads; fewer have no such waits: NVFP4_ERR_UNSUPPORTED),
 * whose waits for keys are made to give up after their limit, by barriers that expect one arrival too
 * many; with NVFP4_KV_STARVE_VALUES added to `causal` the waits for values instead.  status_dev (required) gets bit 4
 * (16), out is not written by the blocks that gave up (what is joined from the workspace is undefined) and the CUDA
 * context stays usable.
 */
#define NVFP4_KV_STARVE_VALUES 2
nvfp4_status nvfp4_kv_selftest_wait_timeout(const nvfp4_kv_cache* cache, const void* q, int64_t q_token, int64_t q_head,
                                            int64_t tokens, int q_heads, const int32_t* table, int64_t table_ld,
                                            int64_t width, const int32_t* lens, const int32_t* offsets, int64_t batch,
                                            int64_t max_q, float scale, int causal, void* out, int64_t out_token,
                                            int64_t out_head, float* lse, int* status_dev, void* workspace,
                                            size_t ws_bytes, void* stream);

/*
 * The same as nvfp4_kv_attention for a batch that shares a prefix: every query also sees the first *prefix_len
 * tokens of the pages prefix[0 .. prefix_width), before its own sequence's (prefix_width * page at most 2^31 - 2048;
 * table, lens, offsets and the causal rule as above; a sequence may have no tokens of its own cached).
 * The prefix's keys and values are read once for all queries of the batch.
 */
nvfp4_status nvfp4_kv_attention_prefix(const nvfp4_kv_cache* cache, const void* q, int64_t q_token, int64_t q_head,
                                       int64_t tokens, int q_heads, const int32_t* prefix, int64_t prefix_width,
                                       const int32_t* prefix_len, const int32_t* table, int64_t table_ld, int64_t width,
                                       const int32_t* lens, const int32_t* offsets, int64_t batch, int64_t max_q,
                                       float scale, int causal, void* out, int64_t out_token, int64_t out_head,
                                       float* lse, int* status_dev, void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* NVFP4KV_H */

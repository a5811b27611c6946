// Host side of include/nvfp4kv.h: argument, alignment and overlap checks (all before any
// launch), then dispatch.  As in api.cu nothing allocates, frees or synchronises.
#include <climits>
#include <cmath>
#include <cstdint>

#include <cuda_runtime.h>

#include "host_checks.h"
#include "kv_kernels.h"
#include "nvfp4kv.h"

using namespace nvfp4;

namespace {

constexpr int64_t kMaxTokens = INT_MAX;
constexpr int kMaxHeads = 65535;
constexpr int64_t kMaxBytes = 1ll << 60;

nvfp4_status result(cudaError_t e) {
    return e == cudaSuccess ? NVFP4_OK : e == cudaErrorNotSupported ? NVFP4_ERR_UNSUPPORTED : NVFP4_ERR_CUDA;
}

// Memory that a call reads and writes: whole extents.
struct Memory {
    struct Span {
        const void* p;
        int64_t n;
    } r[16], w[16];
    int nr = 0, nw = 0;
    void read(const void* p, int64_t n) {
        if (p && n > 0) r[nr++] = Span{p, n};
    }
    void write(const void* p, int64_t n) {
        if (p && n > 0) w[nw++] = Span{p, n};
    }
    nvfp4_status check() const {
        for (int i = 0; i < nw; i++) {
            for (int j = 0; j < nr; j++)
                if (overlap(w[i].p, w[i].n, r[j].p, r[j].n)) return NVFP4_ERR_INVALID_ARG;
            for (int j = i + 1; j < nw; j++)
                if (overlap(w[i].p, w[i].n, w[j].p, w[j].n)) return NVFP4_ERR_INVALID_ARG;
        }
        for (int i = 0; i < nw; i++)
            if (!device_accessible(w[i].p)) return NVFP4_ERR_INVALID_ARG;
        for (int i = 0; i < nr; i++)
            if (!device_accessible(r[i].p)) return NVFP4_ERR_INVALID_ARG;
        return NVFP4_OK;
    }
};

// A strided [tokens, heads, dim] tensor: its strides keep elements apart, its extent in bytes.
struct Extent {
    kv::Tensor t;
    int64_t tokens, heads, dim, esize, bytes;
};
nvfp4_status check_tensor(const void* p, int64_t token, int64_t head, int64_t tokens, int64_t heads, int64_t dim,
                          int64_t esize, Extent* x) {
    if (!p || token < 0 || head < 0) return NVFP4_ERR_INVALID_ARG;
    if (heads > 1 && head < dim) return NVFP4_ERR_INVALID_ARG;
    int64_t across, all;
    if (!mul_ok(heads - 1, head, &across) || !mul_ok(tokens - 1, token, &all)) return NVFP4_ERR_RANGE;
    // heads of a token side by side, or tokens of a head
    if (tokens > 1 && token < across + dim && !(token >= dim && head >= all + dim)) return NVFP4_ERR_INVALID_ARG;
    if (across > kMaxBytes / 8 || all > kMaxBytes / 8) return NVFP4_ERR_RANGE;
    if (!aligned(p, (uintptr_t)esize)) return NVFP4_ERR_ALIGNMENT;
    const auto whole = [&](int64_t n) {
        return aligned(p, (uintptr_t)n) && (token % (n / esize) == 0 || tokens == 1) && (head % (n / esize) == 0 || heads == 1);
    };
    x->t = kv::Tensor{const_cast<void*>(p), token, head, whole(32) ? 2 : whole(16) ? 1 : 0};
    x->tokens = tokens;
    x->heads = heads;
    x->dim = dim;
    x->esize = esize;
    x->bytes = (across + all + dim) * esize;
    return NVFP4_OK;
}

// Whether one lies between the rows of the other: both of one token stride, and each token's heads beside the
// other's (columns of one buffer, a projection's queries, keys and values).
bool beside(const Extent& a, const Extent& b) {
    if (a.esize != b.esize || a.tokens < 2 || b.tokens < 2 || a.t.token != b.t.token) return false;
    const int64_t stride = a.t.token * a.esize;
    const int64_t wa = ((a.heads - 1) * a.t.head + a.dim) * a.esize, wb = ((b.heads - 1) * b.t.head + b.dim) * b.esize;
    if (wa > stride || wb > stride) return false;
    int64_t at = (int64_t)(reinterpret_cast<uintptr_t>(b.t.p) - reinterpret_cast<uintptr_t>(a.t.p)) % stride;
    if (at < 0) at += stride;
    return at >= wa && at + wb <= stride;
}
bool apart(const Extent& a, const Extent& b) { return !overlap(a.t.p, a.bytes, b.t.p, b.bytes) || beside(a, b); }

nvfp4_status check_cache(const nvfp4_kv_cache* c, kv::Cache* out, int64_t* codes, int64_t* sf) {
    if (!c) return NVFP4_ERR_INVALID_ARG;
    if (c->dim != 64 && c->dim != 128) return NVFP4_ERR_UNSUPPORTED;
    if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1))) return NVFP4_ERR_UNSUPPORTED;
    if (c->pages < 0 || c->heads < 1) return NVFP4_ERR_INVALID_ARG;
    if (c->heads > kMaxHeads || c->pages > INT_MAX) return NVFP4_ERR_RANGE;
    int64_t rows;
    if (!mul_ok(c->pages, (int64_t)c->heads * 2 * c->page, &rows) || rows > kMaxBytes / c->dim) return NVFP4_ERR_RANGE;
    *codes = rows * (c->dim / 2);
    *sf = rows * (c->dim / 16);
    if (c->pages > 0 && (!c->codes || !c->sf)) return NVFP4_ERR_INVALID_ARG;
    if (!c->S_k || !c->S_v) return NVFP4_ERR_INVALID_ARG;
    if (!aligned(c->codes, 16) || !aligned(c->sf, 16) || !aligned(c->S_k, 4) || !aligned(c->S_v, 4))
        return NVFP4_ERR_ALIGNMENT;
    int log2 = 4;
    while ((1 << log2) < c->page) log2++;
    *out = kv::Cache{c->codes, c->sf, c->S_k, c->S_v, c->pages, log2, c->heads, c->dim};
    return NVFP4_OK;
}

nvfp4_status check_table(const int32_t* table, int64_t ld, int64_t width, int64_t batch, int page, Memory* mem) {
    if (batch < 0 || width < 0 || (batch > 1 && ld < width)) return NVFP4_ERR_INVALID_ARG;
    if (batch > kMaxTokens || width > INT_MAX / page) return NVFP4_ERR_RANGE;
    if (batch == 0 || width == 0) return NVFP4_OK;
    if (!table) return NVFP4_ERR_INVALID_ARG;
    if (!aligned(table, 4)) return NVFP4_ERR_ALIGNMENT;
    int64_t rows;
    if (!mul_ok(batch - 1, ld, &rows) || rows > kMaxBytes / 8) return NVFP4_ERR_RANGE;
    mem->read(table, (rows + width) * 4);
    return NVFP4_OK;
}

}  // namespace

extern "C" {

nvfp4_status nvfp4_rope_turns(int rot, double base, nvfp4_rope_scaling scaling, double factor, double original_len,
                              double slow, double fast, uint64_t* turns) {
    if (!turns || rot < 2 || rot > 1024 || rot % 2 || !(base > 1.0) || !std::isfinite(base)) return NVFP4_ERR_INVALID_ARG;
    if (scaling < NVFP4_ROPE_PLAIN || scaling > NVFP4_ROPE_BANDS) return NVFP4_ERR_INVALID_ARG;
    if (scaling != NVFP4_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return NVFP4_ERR_INVALID_ARG;
    if (scaling == NVFP4_ROPE_BANDS &&
        (!(original_len > 0.0) || !std::isfinite(original_len) || !(slow >= 0.0) || !(fast > slow) || !std::isfinite(fast)))
        return NVFP4_ERR_INVALID_ARG;
    if (scaling == NVFP4_ROPE_BASE) {
        if (rot == 2) return NVFP4_ERR_INVALID_ARG;
        base *= std::pow(factor, (double)rot / (rot - 2));
        if (!std::isfinite(base)) return NVFP4_ERR_RANGE;
    }
    const double pi = 3.14159265358979323846;
    for (int i = 0; i < rot / 2; i++) {
        double f = std::pow(base, -2.0 * i / rot) / (2.0 * pi);
        if (scaling == NVFP4_ROPE_LINEAR) f /= factor;
        if (scaling == NVFP4_ROPE_BANDS) {
            double g = (original_len * f - slow) / (fast - slow);
            g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
            f *= (1.0 - g) / factor + g;
        }
        turns[i] = (uint64_t)std::nearbyint(std::ldexp(f, 64));  // f < 1/6
    }
    return NVFP4_OK;
}

nvfp4_status nvfp4_rope(const void* x, int64_t x_token, int64_t x_head, void* out, int64_t out_token, int64_t out_head,
                        nvfp4_dtype dt, int64_t tokens, int heads, int dim, int rot, const int64_t* positions,
                        const uint64_t* turns, float magnitude, nvfp4_rope_layout layout, int inverse, void* stream) {
    if ((dt != NVFP4_IN_BF16 && dt != NVFP4_IN_F32) || tokens < 0 || heads < 0 || dim < 0 || rot < 0) return NVFP4_ERR_INVALID_ARG;
    if (layout != NVFP4_ROPE_NEIGHBOURS && layout != NVFP4_ROPE_HALVES) return NVFP4_ERR_INVALID_ARG;
    if (dim % 2 || rot % 2 || rot > dim || !std::isfinite(magnitude)) return NVFP4_ERR_INVALID_ARG;
    if (tokens > kMaxTokens || heads > kMaxHeads || dim > 1024) return NVFP4_ERR_RANGE;
    if (tokens == 0 || heads == 0 || dim == 0) return NVFP4_OK;
    const int64_t esize = dt == NVFP4_IN_BF16 ? 2 : 4;
    Extent a, b;
    nvfp4_status st;
    if ((st = check_tensor(x, x_token, x_head, tokens, heads, dim, esize, &a)) != NVFP4_OK ||
        (st = check_tensor(out, out_token, out_head, tokens, heads, dim, esize, &b)) != NVFP4_OK)
        return st;
    if (rot > 0 && (!positions || !turns)) return NVFP4_ERR_INVALID_ARG;
    if (!aligned(positions, 8) || !aligned(turns, 8)) return NVFP4_ERR_ALIGNMENT;
    const bool in_place = x == out;
    if (in_place && ((tokens > 1 && x_token != out_token) || (heads > 1 && x_head != out_head))) return NVFP4_ERR_INVALID_ARG;
    if (!in_place && !apart(a, b)) return NVFP4_ERR_INVALID_ARG;
    if (in_place && rot == 0) return device_accessible(x) ? NVFP4_OK : NVFP4_ERR_INVALID_ARG;
    Memory mem;
    if (rot > 0) {
        mem.read(positions, tokens * 8);
        mem.read(turns, rot / 2 * 8);
    }
    mem.write(out, b.bytes);
    if ((st = mem.check()) != NVFP4_OK) return st;
    if (!device_accessible(x)) return NVFP4_ERR_INVALID_ARG;
    const int sms = sm_count();
    if (sms <= 0) return NVFP4_ERR_CUDA;
    kv::Rope p = {};
    p.x = a.t;
    p.out = b.t;
    p.dtype = dt == NVFP4_IN_BF16 ? 0 : 1;
    p.heads = heads;
    p.dim = dim;
    p.rot = rot;
    p.halves = layout == NVFP4_ROPE_HALVES;
    p.inverse = inverse != 0;
    p.tokens = tokens;
    p.positions = positions;
    p.turns = turns;
    p.magnitude = magnitude;
    return result(kv::launch_rope(p, sms, static_cast<cudaStream_t>(stream)));
}

nvfp4_status nvfp4_kv_write(const nvfp4_kv_cache* cache, const void* k, int64_t k_token, int64_t k_head, const void* v,
                            int64_t v_token, int64_t v_head, nvfp4_dtype dt, int64_t tokens, const int64_t* slots,
                            nvfp4_kv_method method, int* status_dev, void* stream) {
    if ((dt != NVFP4_IN_BF16 && dt != NVFP4_IN_F32) || (method != NVFP4_KV_ABSMAX && method != NVFP4_KV_SWEEP) || tokens < 0)
        return NVFP4_ERR_INVALID_ARG;
    kv::Write p = {};
    int64_t codes, sf;
    nvfp4_status st = check_cache(cache, &p.c, &codes, &sf);
    if (st != NVFP4_OK) return st;
    if (tokens > kMaxTokens) return NVFP4_ERR_RANGE;
    if (tokens == 0) return NVFP4_OK;
    if ((!k && !v) || !slots) return NVFP4_ERR_INVALID_ARG;
    const int64_t esize = dt == NVFP4_IN_BF16 ? 2 : 4;
    Memory mem;
    Extent x[2];
    const void* in[2] = {k, v};
    const int64_t token[2] = {k_token, v_token}, head[2] = {k_head, v_head};
    for (int i = 0; i < 2; i++) {
        if (!in[i]) continue;
        if ((st = check_tensor(in[i], token[i], head[i], tokens, p.c.heads, p.c.dim, esize, &x[i])) != NVFP4_OK) return st;
        p.in[i] = x[i].t;
        mem.read(in[i], x[i].bytes);
    }
    if (!aligned(slots, 8) || !aligned(status_dev, 4)) return NVFP4_ERR_ALIGNMENT;
    mem.read(slots, tokens * 8);
    mem.read(p.c.S_k, 4);
    mem.read(p.c.S_v, 4);
    mem.write(p.c.codes, codes);
    mem.write(p.c.sf, sf);
    mem.write(status_dev, 4);
    if ((st = mem.check()) != NVFP4_OK) return st;
    const int sms = sm_count();
    if (sms <= 0) return NVFP4_ERR_CUDA;
    p.dtype = dt == NVFP4_IN_BF16 ? 0 : 1;
    p.method = method == NVFP4_KV_SWEEP ? 0 : 1;
    p.tokens = tokens;
    p.slots = slots;
    p.status = status_dev;
    return result(kv::launch_write(p, sms, static_cast<cudaStream_t>(stream)));
}

nvfp4_status nvfp4_kv_read(const nvfp4_kv_cache* cache, const int32_t* table, int64_t table_ld, int64_t width,
                           const int32_t* starts, const int32_t* offsets, int64_t batch, void* k, int64_t k_token,
                           int64_t k_head, void* v, int64_t v_token, int64_t v_head, nvfp4_dtype out_dt, int64_t tokens,
                           int* status_dev, void* stream) {
    if ((out_dt != NVFP4_IN_BF16 && out_dt != NVFP4_IN_F32) || tokens < 0) return NVFP4_ERR_INVALID_ARG;
    kv::Read p = {};
    int64_t codes, sf;
    Memory mem;
    nvfp4_status st = check_cache(cache, &p.c, &codes, &sf);
    if (st != NVFP4_OK) return st;
    if ((st = check_table(table, table_ld, width, batch, cache->page, &mem)) != NVFP4_OK) return st;
    if (tokens > kMaxTokens) return NVFP4_ERR_RANGE;
    if (tokens == 0 || batch == 0) return NVFP4_OK;
    if ((!k && !v) || !offsets) return NVFP4_ERR_INVALID_ARG;
    const int64_t esize = out_dt == NVFP4_IN_BF16 ? 2 : 4;
    Extent x[2];
    void* out[2] = {k, v};
    const int64_t token[2] = {k_token, v_token}, head[2] = {k_head, v_head};
    for (int i = 0; i < 2; i++) {
        if (!out[i]) continue;
        if ((st = check_tensor(out[i], token[i], head[i], tokens, p.c.heads, p.c.dim, esize, &x[i])) != NVFP4_OK) return st;
        p.out[i] = x[i].t;
    }
    if (k && v && !apart(x[0], x[1])) return NVFP4_ERR_INVALID_ARG;
    if (!aligned(offsets, 4) || !aligned(starts, 4) || !aligned(status_dev, 4)) return NVFP4_ERR_ALIGNMENT;
    mem.read(p.c.codes, codes);
    mem.read(p.c.sf, sf);
    mem.read(p.c.S_k, 4);
    mem.read(p.c.S_v, 4);
    mem.read(offsets, (batch + 1) * 4);
    mem.read(starts, batch * 4);
    mem.write(status_dev, 4);
    Memory second = mem;                                         // k and v may be columns of one buffer
    if (k) mem.write(k, x[0].bytes);
    if (v) second.write(v, x[1].bytes);
    if ((st = mem.check()) != NVFP4_OK || (st = second.check()) != NVFP4_OK) return st;
    const int sms = sm_count();
    if (sms <= 0) return NVFP4_ERR_CUDA;
    p.dtype = out_dt == NVFP4_IN_BF16 ? 0 : 1;
    p.table = table;
    p.starts = starts;
    p.offsets = offsets;
    p.table_ld = table_ld;
    p.width = width;
    p.batch = batch;
    p.tokens = tokens;
    p.status = status_dev;
    return result(kv::launch_read(p, sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"

namespace {

// Sizes of a call, if they are ones that a call takes.
nvfp4_status attention_sizes(const nvfp4_kv_cache* c, int64_t tokens, int q_heads, int64_t batch, int64_t width, int64_t max_q,
                             int64_t prefix_width, kv::Sizes* s) {
    if (tokens < 0 || batch < 0 || width < 0 || max_q < 0 || prefix_width < 0) return NVFP4_ERR_INVALID_ARG;
    if (q_heads < 1 || q_heads % c->heads) return NVFP4_ERR_INVALID_ARG;
    if (q_heads > kMaxHeads || tokens > kMaxTokens || batch > kMaxTokens || max_q > kMaxTokens) return NVFP4_ERR_RANGE;
    if (width > kv::kMaxLength / c->page || prefix_width > kv::kMaxLength / c->page) return NVFP4_ERR_RANGE;
    if (max_q > tokens) max_q = tokens;
    *s = kv::Sizes{tokens, batch, max_q, q_heads, c->heads, c->dim, width * c->page, prefix_width * c->page};
    return NVFP4_OK;
}

nvfp4_status attention(const nvfp4_kv_cache* cache, const void* q, int64_t q_token, int64_t q_head, int64_t tokens, int q_heads,
                       bool shared, const int32_t* prefix, int64_t prefix_width, const int32_t* prefix_len,
                       const int32_t* table, int64_t table_ld, int64_t width, const int32_t* lens, const int32_t* offsets,
                       int64_t batch, int64_t max_q, float scale, int causal, void* out, int64_t out_token, int64_t out_head,
                       float* lse, int* status_dev, void* workspace, size_t ws_bytes, int starve, void* stream) {
    kv::Attention p = {};
    kv::Sizes s;
    int64_t codes, sf;
    Memory mem;
    nvfp4_status st = check_cache(cache, &p.c, &codes, &sf);
    if (st != NVFP4_OK || (st = attention_sizes(cache, tokens, q_heads, batch, width, max_q, prefix_width, &s)) != NVFP4_OK)
        return st;
    if (!(scale >= 0.0f) || !std::isfinite(scale)) return NVFP4_ERR_INVALID_ARG;
    if ((st = check_table(table, table_ld, width, batch, cache->page, &mem)) != NVFP4_OK) return st;
    if (shared && (st = check_table(prefix, prefix_width, prefix_width, 1, cache->page, &mem)) != NVFP4_OK) return st;
    if (tokens == 0 || batch == 0 || s.max_q == 0) return NVFP4_OK;
    if (!lens || !offsets || (shared && !prefix_len)) return NVFP4_ERR_INVALID_ARG;
    Extent a, b;
    if ((st = check_tensor(q, q_token, q_head, tokens, q_heads, p.c.dim, 2, &a)) != NVFP4_OK ||
        (st = check_tensor(out, out_token, out_head, tokens, q_heads, p.c.dim, 2, &b)) != NVFP4_OK)
        return st;
    if (!apart(a, b)) return NVFP4_ERR_INVALID_ARG;
    p.plan = kv::make_plan(s);
    if (!p.plan.fits()) return NVFP4_ERR_RANGE;
    if (starve && p.plan.own.rows < kv::kTileRows) return NVFP4_ERR_UNSUPPORTED;
    if (p.plan.bytes > 0 && (!workspace || ws_bytes < (size_t)p.plan.bytes)) return NVFP4_ERR_INVALID_ARG;
    if (p.plan.bytes == 0) workspace = nullptr;
    if (!aligned(lens, 4) || !aligned(offsets, 4) || !aligned(prefix_len, 4) || !aligned(lse, 4) || !aligned(status_dev, 4) ||
        !aligned(workspace, 256))
        return NVFP4_ERR_ALIGNMENT;
    mem.read(p.c.codes, codes);
    mem.read(p.c.sf, sf);
    mem.read(p.c.S_k, 4);
    mem.read(p.c.S_v, 4);
    mem.read(lens, batch * 4);
    mem.read(offsets, (batch + 1) * 4);
    if (shared) mem.read(prefix_len, 4);
    mem.write(out, b.bytes);
    mem.write(lse, tokens * q_heads * 4);
    mem.write(status_dev, 4);
    mem.write(workspace, p.plan.bytes);
    if ((st = mem.check()) != NVFP4_OK) return st;
    // q, which may lie beside out in one buffer, against the others
    Memory rest;
    rest.read(q, a.bytes);
    rest.write(lse, tokens * q_heads * 4);
    rest.write(status_dev, 4);
    rest.write(workspace, p.plan.bytes);
    if ((st = rest.check()) != NVFP4_OK) return st;
    if (sm_count() <= 0) return NVFP4_ERR_CUDA;
    p.q = a.t;
    p.out = b.t;
    p.q_heads = q_heads;
    p.group = q_heads / p.c.heads;
    p.causal = causal != 0;
    p.tokens = tokens;
    p.batch = batch;
    p.max_q = s.max_q;
    p.table = table;
    p.lens = lens;
    p.offsets = offsets;
    p.table_ld = table_ld;
    p.width = p.c.pages > 0 ? width : 0;                         // an empty pool holds nothing
    p.prefix = prefix;
    p.prefix_len = shared ? prefix_len : nullptr;
    p.prefix_width = p.c.pages > 0 ? prefix_width : 0;
    p.scale = scale;
    p.lse = lse;
    p.status = status_dev;
    p.workspace = workspace;
    p.starve = starve;
    return result(kv::launch_attention(p, static_cast<cudaStream_t>(stream)));
}

}  // namespace

extern "C" {

size_t nvfp4_kv_attention_workspace(const nvfp4_kv_cache* cache, int64_t tokens, int q_heads, int64_t batch,
                                    int64_t width, int64_t max_q, int64_t prefix_width) {
    kv::Sizes s;
    if (!cache || (cache->dim != 64 && cache->dim != 128) || cache->page < 16 || cache->page > 1024 || cache->heads < 1)
        return 0;
    if (attention_sizes(cache, tokens, q_heads, batch, width, max_q, prefix_width, &s) != NVFP4_OK) return 0;
    if (tokens == 0 || batch == 0 || s.max_q == 0) return 0;
    const kv::Plan p = kv::make_plan(s);
    return p.fits() ? (size_t)p.bytes : 0;
}

nvfp4_status nvfp4_kv_attention(const nvfp4_kv_cache* cache, const void* q, int64_t q_token, int64_t q_head,
                                int64_t tokens, int q_heads, const int32_t* table, int64_t table_ld, int64_t width,
                                const int32_t* lens, const int32_t* offsets, int64_t batch, int64_t max_q, float scale,
                                int causal, void* out, int64_t out_token, int64_t out_head, float* lse, int* status_dev,
                                void* workspace, size_t ws_bytes, void* stream) {
    return attention(cache, q, q_token, q_head, tokens, q_heads, false, nullptr, 0, nullptr, table, table_ld, width, lens, offsets,
                     batch, max_q, scale, causal, out, out_token, out_head, lse, status_dev, workspace, ws_bytes, 0, stream);
}

nvfp4_status nvfp4_kv_selftest_wait_timeout(const nvfp4_kv_cache* cache, const void* q, int64_t q_token, int64_t q_head,
                                            int64_t tokens, int q_heads, const int32_t* table, int64_t table_ld, int64_t width,
                                            const int32_t* lens, const int32_t* offsets, int64_t batch, int64_t max_q,
                                            float scale, int causal, void* out, int64_t out_token, int64_t out_head, float* lse,
                                            int* status_dev, void* workspace, size_t ws_bytes, void* stream) {
    if (!status_dev) return NVFP4_ERR_INVALID_ARG;
    return attention(cache, q, q_token, q_head, tokens, q_heads, false, nullptr, 0, nullptr, table, table_ld, width, lens, offsets,
                     batch, max_q, scale, causal & ~NVFP4_KV_STARVE_VALUES, out, out_token, out_head, lse, status_dev, workspace, ws_bytes,
                     causal & NVFP4_KV_STARVE_VALUES ? 2 : 1, stream);
}

nvfp4_status nvfp4_kv_attention_prefix(const nvfp4_kv_cache* cache, const void* q, int64_t q_token, int64_t q_head,
                                       int64_t tokens, int q_heads, const int32_t* prefix, int64_t prefix_width,
                                       const int32_t* prefix_len, const int32_t* table, int64_t table_ld, int64_t width,
                                       const int32_t* lens, const int32_t* offsets, int64_t batch, int64_t max_q,
                                       float scale, int causal, void* out, int64_t out_token, int64_t out_head,
                                       float* lse, int* status_dev, void* workspace, size_t ws_bytes, void* stream) {
    return attention(cache, q, q_token, q_head, tokens, q_heads, true, prefix, prefix_width, prefix_len, table, table_ld, width,
                     lens, offsets, batch, max_q, scale, causal, out, out_token, out_head, lse, status_dev, workspace, ws_bytes,
                     0, stream);
}

}  // extern "C"

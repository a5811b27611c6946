// Rotary positions of query and key heads, and their transpose (nvfp4_rope).
//
// Angles: a frequency is a fraction of a turn in 64-bit fixed point, so position * frequency
// modulo 2^64 is the angle modulo a turn without error, for any position; its upper 32 bits
// as a signed number of 2^-31 half-turns go to sincospif.  The conversion to fp32 rounds by up to 2^-25
// of the angle's half-turns, the same order as the function's own error.
//
// A block takes a few tokens: its threads compute the sines of each pair once, into shared memory, while
// the elements are on their way.  A thread owns one unit of a head -- V pairs, in two pieces of 16 bytes, either one
// in each half of the pairs or of whole pairs, so that neighbouring threads' pieces are neighbours -- in up to kHeads heads.
//
// Bound by memory: 8192 tokens of 40 heads of 128 in bf16, 168 MB, in 27.5 us, 6.1 TB/s (a copy: 6.7).  Sines computed by
// every thread for itself took 33.6, four heads a thread instead of two 31.7.
#include "kv_kernels.h"
#include "nvfp4_device.cuh"

namespace nvfp4 {
namespace kv {
namespace {

constexpr int kThreads = 256, kHeads = 2;

// V elements of type DT: one 16-byte access, or single elements (V = 1).
template <int DT, int V>
struct Words {
    static constexpr int N = V == 1 ? 1 : 4;
    uint32_t w[N];
};
template <int DT, int V>
__device__ __forceinline__ Words<DT, V> load(const void* base, int64_t e) {
    Words<DT, V> r;
    if constexpr (V == 1) {
        r.w[0] = DT == 0 ? (uint32_t)static_cast<const uint16_t*>(base)[e] : static_cast<const uint32_t*>(base)[e];
    } else {
        const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const char*>(base) + e * (DT == 0 ? 2 : 4));
        r.w[0] = v.x, r.w[1] = v.y, r.w[2] = v.z, r.w[3] = v.w;
    }
    return r;
}
template <int DT, int V>
__device__ __forceinline__ void store(void* base, int64_t e, const Words<DT, V>& r) {
    if constexpr (V == 1) {
        if (DT == 0) static_cast<uint16_t*>(base)[e] = (uint16_t)r.w[0];
        else static_cast<uint32_t*>(base)[e] = r.w[0];
    } else {
        *reinterpret_cast<uint4*>(static_cast<char*>(base) + e * (DT == 0 ? 2 : 4)) =
            make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    }
}
template <int DT, int V>
__device__ __forceinline__ float get(const Words<DT, V>& r, int i) {
    if (DT != 0) return __uint_as_float(r.w[i]);
    if (V == 1) return bf16lo(r.w[0]);
    return i & 1 ? bf16hi(r.w[i / 2]) : bf16lo(r.w[i / 2]);
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int DT, int V>
__device__ __forceinline__ void pack(const float (&v)[V], Words<DT, V>& r) {
#pragma unroll
    for (int i = 0; i < Words<DT, V>::N; i++) {
        if (DT != 0) r.w[i] = __float_as_uint(v[i]);
        else if (V == 1) r.w[0] = bf16x2(v[0], 0.0f);
        else r.w[i] = bf16x2(v[(2 * i) % V], v[(2 * i + 1) % V]);
    }
}

// Block (units of a head, heads, tokens); heads y, y + hl, ... of a thread.
template <int DT, int V, int HALVES>
__global__ void __launch_bounds__(kThreads) rope_kernel(Rope p, int hl, int copy) {
    extern __shared__ float2 s_turn[];                           // [tokens][rot / 2]: magnitude times cosine and sine
    grid_launch_dependents();
    grid_dependency_wait();
    const int64_t token0 = (int64_t)blockIdx.x * blockDim.z, token = token0 + threadIdx.z;
    const int y = blockIdx.y * blockDim.y + threadIdx.y;
    const bool mine = token < p.tokens && y < hl;
    const int half = p.rot / 2, units = half / V;
    constexpr bool kSplit = HALVES || V > 1;                     // else a unit is one pair of neighbours
    const int64_t xt = token * p.x.token, ot = token * p.out.token;
    Words<DT, V> xa[kHeads], xb[kHeads];
    // where a unit's pieces begin
    auto first = [&](int u) { return u >= units ? p.rot + (u - units) * V : kSplit ? u * V : 2 * u; };
    auto second = [&](int u) { return u >= units ? p.rot + (u - units + copy) * V : kSplit ? u * V + half : 2 * u + 1; };
    auto read = [&](int u) {
#pragma unroll
        for (int k = 0; k < kHeads; k++) {
            const int h = y + k * hl;
            if (h < p.heads) {
                xa[k] = load<DT, V>(p.x.p, xt + h * p.x.head + first(u));
                xb[k] = load<DT, V>(p.x.p, xt + h * p.x.head + second(u));
            }
        }
    };
    int u = threadIdx.x;
    const int last = units + copy;
    if (mine && u < last) read(u);
    const int tid = threadIdx.x + blockDim.x * (threadIdx.y + blockDim.y * threadIdx.z);
    const int threads = blockDim.x * blockDim.y * blockDim.z;
    for (int x = tid; x < half * (int)blockDim.z; x += threads) {
        const int z = x / half;
        if (token0 + z < p.tokens) {
            const int hi = (int)(((uint64_t)p.positions[token0 + z] * p.turns[x - z * half]) >> 32);
            float s, c;
            sincospif(__fmul_rn((float)hi, 4.656612873077393e-10f), &s, &c);                // 2^-31
            s_turn[x] = make_float2(c * p.magnitude, s * (p.inverse ? -p.magnitude : p.magnitude));
        }
    }
    __syncthreads();
    if (!mine) return;
    for (; u < last; u += blockDim.x) {
        if (u != (int)threadIdx.x) read(u);
        const bool rotate = u < units;
        float c[V], s[V];
        if (rotate) {
#pragma unroll
            for (int i = 0; i < V; i++) {
                // whole pairs: V / 2 in each piece
                const int pair = HALVES || V == 1 ? u * V + i : (i < V / 2 ? first(u) : second(u) - V) / 2 + i;
                const float2 f = s_turn[threadIdx.z * half + pair];
                c[i] = f.x, s[i] = f.y;
            }
        }
#pragma unroll
        for (int k = 0; k < kHeads; k++) {
            const int h = y + k * hl;
            if (h >= p.heads) break;
            if (rotate) {
                float fa[V], fb[V];
#pragma unroll
                for (int i = 0; i < V; i++) {
                    if (HALVES || V == 1) {
                        const float va = get(xa[k], i), vb = get(xb[k], i);
                        fa[i] = __fmaf_rn(va, c[i], -__fmul_rn(vb, s[i]));
                        fb[i] = __fmaf_rn(va, s[i], __fmul_rn(vb, c[i]));
                    } else {
                        const Words<DT, V>& w = 2 * i < V ? xa[k] : xb[k];
                        const float va = get(w, 2 * i % V), vb = get(w, (2 * i + 1) % V);
                        float* f = 2 * i < V ? fa : fb;
                        f[2 * i % V] = __fmaf_rn(va, c[i], -__fmul_rn(vb, s[i]));
                        f[(2 * i + 1) % V] = __fmaf_rn(va, s[i], __fmul_rn(vb, c[i]));
                    }
                }
                pack<DT, V>(fa, xa[k]);
                pack<DT, V>(fb, xb[k]);
            }
            store<DT, V>(p.out.p, ot + h * p.out.head + first(u), xa[k]);
            store<DT, V>(p.out.p, ot + h * p.out.head + second(u), xb[k]);
        }
    }
}

template <int DT, int V>
cudaError_t launch(const Rope& p, int sms, cudaStream_t s) {
    const bool in_place = p.x.p == p.out.p;
    const int copy = in_place ? 0 : (p.dim - p.rot) / (2 * V);
    const int units = p.rot / (2 * V) + copy;
    // several heads to a thread where that still fills the GPU
    const bool many = p.tokens * units * p.heads >= (int64_t)sms * 2048;
    const int hl = many ? (p.heads + kHeads - 1) / kHeads : p.heads;
    dim3 block, grid;
    block.x = units < kThreads ? units : kThreads;
    block.y = kThreads / block.x < (unsigned)hl ? kThreads / block.x : hl;
    block.z = kThreads / (block.x * block.y);
    if (block.z > 64) block.z = 64;
    if (!many) block.z = 1;
    const size_t smem = (size_t)block.z * (p.rot / 2) * sizeof(float2);      // at most 64 tokens of 2 or 1 of 512 pairs
    grid.x = (unsigned)((p.tokens + block.z - 1) / block.z);
    grid.y = (hl + block.y - 1) / block.y;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return p.halves ? cudaLaunchKernelEx(&cfg, rope_kernel<DT, V, 1>, p, hl, copy)
                    : cudaLaunchKernelEx(&cfg, rope_kernel<DT, V, 0>, p, hl, copy);
}

}  // namespace

cudaError_t launch_rope(const Rope& p, int sms, cudaStream_t s) {
    const int v = p.dtype == 0 ? 8 : 4;
    const bool vec = p.x.vec && p.out.vec && p.rot % (2 * v) == 0 && p.dim % (2 * v) == 0;
    if (p.dtype == 0) return vec ? launch<0, 8>(p, sms, s) : launch<0, 1>(p, sms, s);
    return vec ? launch<1, 4>(p, sms, s) : launch<1, 1>(p, sms, s);
}

}  // namespace kv
}  // namespace nvfp4

// AdamW over many tensors in one launch, states in 32 or in 8 bits; the global norm of their gradients; 8-bit states as f32.
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// All of it is bound by memory: 28 bytes an element with f32 parameters, gradients and states, 10 with 16-bit ones and 8-bit states.
// The tensors' table travels in the launch's arguments (no copy to the device, nothing to keep), a block finds its chunk's tensor by bisection.
//
// States in 8 bits, in blocks of 256 elements, the share of a warp (eight elements a lane).  m: sign, 4 exponent and 3 mantissa bits;
// v: 5 exponent and 3 mantissa bits (a second moment spans the square of a first one's range); each times a scale of its block, so that
// the largest gets the largest code.  A code is the upper bits of an f32 number whose exponents were moved down to where the
// code's begin: below them f32 is as evenly spaced as the code, so that coding is one multiplication, an addition and a shift, subnormal values
// included.  What the shift drops decides the rounding: half of it added is rounding to nearest (halves up), 16 random bits added make
// the mean of the code the value.  Rounded to nearest, b2 = 0.999 could not move a v with steps of an eighth; at random it moves on average
// as it should.  v above 0 never becomes 0, so that no update is divided by eps alone.
// Products and sums are rounded one by one (no contraction): which of two codes a value gets hangs on its last bit, and is the same wherever
// the formulas are evaluated in f32.
#include "adamw.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstring>

namespace ow {

typedef __nv_bfloat16 bf16;

constexpr int THREADS_W = 256, PASS = 8 * THREADS_W, CHUNK = 2 * PASS;
constexpr float TOP_M = 480.f, TOP_V = 61440.f, LEAST = 1e-30f;
constexpr float DOWN_M = 0x1p-120f, UP_M = 0x1p120f, DOWN_V = 0x1p-111f, UP_V = 0x1p111f;

struct Item {
    void *param;
    bf16 *copy;
    const void *grad;
    void *m, *v;
    float *scales;
    int64_t numel;
    uint32_t first;                        // chunk
    uint16_t ptype, gtype;
};
static_assert(sizeof(Item) == 64, "the table's rows");

struct Hyper {
    float b1, c1, b2, c2, eps, decay, a, s2;
    float max_norm;
    uint32_t seed, step;
    const float *norm, *lr_dev;
    const int32_t *step_dev;
    double b1d, b2d, lr, wd;
    int32_t seeded;
};

template <int CAP> struct Table {
    Hyper h;
    int32_t n, number;                     // tensors; the first one's number in the call
    Item t[CAP];
};

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {     // an integer hash
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}

// Eight values of a lane: side by side (VEC), or 32 apart, those below n.
template <bool VEC> __device__ __forceinline__ int64_t place(int64_t base, int lane, int k) { return base + (VEC ? lane * 8 + k : lane + 32 * k); }

template <bool VEC> __device__ __forceinline__ void load(const void *p, int type, int64_t base, int lane, int64_t n, float (&x)[8]) {
    if (type == PACER_F32) {
        const float *q = reinterpret_cast<const float *>(p);
        if (VEC) {
            const float4 u = *reinterpret_cast<const float4 *>(q + base + lane * 8), w = *reinterpret_cast<const float4 *>(q + base + lane * 8 + 4);
            x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
        } else
#pragma unroll
            for (int k = 0; k < 8; ++k) { const int64_t i = place<false>(base, lane, k); x[k] = i < n ? q[i] : 0.f; }
    } else {
        uint32_t h[8];
        const uint16_t *q = reinterpret_cast<const uint16_t *>(p);
        if (VEC) {
            const uint4 u = *reinterpret_cast<const uint4 *>(q + base + lane * 8);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) h[k] = k & 1 ? w[k >> 1] >> 16 : w[k >> 1] & 0xffffu;
        } else
#pragma unroll
            for (int k = 0; k < 8; ++k) { const int64_t i = place<false>(base, lane, k); h[k] = i < n ? q[i] : 0u; }
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = type == PACER_BF16 ? __uint_as_float(h[k] << 16) : __half2float(__ushort_as_half((unsigned short)h[k]));
    }
}
template <bool VEC> __device__ __forceinline__ void store(float *q, int64_t base, int lane, int64_t n, const float (&x)[8]) {
    if (VEC) {
        *reinterpret_cast<float4 *>(q + base + lane * 8) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4 *>(q + base + lane * 8 + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else
#pragma unroll
        for (int k = 0; k < 8; ++k) { const int64_t i = place<false>(base, lane, k); if (i < n) q[i] = x[k]; }
}
// h: eight 16-bit patterns
template <bool VEC> __device__ __forceinline__ void store16(bf16 *p, int64_t base, int lane, int64_t n, const uint32_t (&h)[8]) {
    uint16_t *q = reinterpret_cast<uint16_t *>(p);
    if (VEC) *reinterpret_cast<uint4 *>(q + base + lane * 8) = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
    else
#pragma unroll
        for (int k = 0; k < 8; ++k) { const int64_t i = place<false>(base, lane, k); if (i < n) q[i] = (uint16_t)h[k]; }
}
template <bool VEC> __device__ __forceinline__ void load_codes(const uint8_t *q, int64_t base, int lane, int64_t n, uint32_t (&c)[8]) {
    if (VEC) {
        const uint2 u = *reinterpret_cast<const uint2 *>(q + base + lane * 8);
#pragma unroll
        for (int k = 0; k < 8; ++k) c[k] = ((k < 4 ? u.x : u.y) >> (8 * (k & 3))) & 0xffu;
    } else
#pragma unroll
        for (int k = 0; k < 8; ++k) { const int64_t i = place<false>(base, lane, k); c[k] = i < n ? q[i] : 0u; }
}
template <bool VEC> __device__ __forceinline__ void store_codes(uint8_t *q, int64_t base, int lane, int64_t n, const uint32_t (&c)[8]) {
    if (VEC) *reinterpret_cast<uint2 *>(q + base + lane * 8) = make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
    else
#pragma unroll
        for (int k = 0; k < 8; ++k) { const int64_t i = place<false>(base, lane, k); if (i < n) q[i] = (uint8_t)c[k]; }
}

__device__ __forceinline__ float value_m(uint32_t c, float scale) { return __fmul_rn(__uint_as_float((c & 0x7fu) << 20 | (c & 0x80u) << 24) * UP_M, scale); }
__device__ __forceinline__ float value_v(uint32_t c, float scale) { return __fmul_rn(__uint_as_float(c << 20) * UP_V, scale); }

// The scale of a block from its largest bits (NaN above all, so that a block with one is NaN from then on).
__device__ __forceinline__ void scale_of(uint32_t bits, float top, float one_by_top, float &scale, float &inverse) {
    const float peak = __uint_as_float(bits);
    const bool none = peak <= LEAST;       // too small to be told from 0: codes and scale are 0
    scale = none ? 0.f : __fmul_rn(peak, one_by_top);
    inverse = none ? 0.f : __fdiv_rn(top, peak);
}

// Eight elements of one lane, all of a warp 256: a block of 8-bit states.  seed: the tensor's.
template <int BITS, bool VEC>
__device__ __forceinline__ void update(const Item &t, const Hyper &h, float a, float s2, float decay, float clip, bool clipped, uint32_t key, int64_t base, int lane) {
    const int64_t n = t.numel;
    float p[8], g[8], m[8], v[8];
    uint32_t cm[8], cv[8];
    load<VEC>(t.grad, t.gtype, base, lane, n, g);
    load<VEC>(t.param, t.ptype, base, lane, n, p);
    if (BITS == 32) {
        load<VEC>(t.m, PACER_F32, base, lane, n, m);
        load<VEC>(t.v, PACER_F32, base, lane, n, v);
    } else {
        load_codes<VEC>(reinterpret_cast<const uint8_t *>(t.m), base, lane, n, cm);
        load_codes<VEC>(reinterpret_cast<const uint8_t *>(t.v), base, lane, n, cv);
        const float2 s = *reinterpret_cast<const float2 *>(t.scales + (base >> 8) * 2);
#pragma unroll
        for (int k = 0; k < 8; ++k) { m[k] = value_m(cm[k], s.x); v[k] = value_v(cv[k], s.y); }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (clipped) g[k] = __fmul_rn(g[k], clip);
        m[k] = __fadd_rn(__fmul_rn(m[k], h.b1), __fmul_rn(g[k], h.c1));
        v[k] = __fadd_rn(__fmul_rn(v[k], h.b2), __fmul_rn(__fmul_rn(g[k], g[k]), h.c2));
        float root, share;
        asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v[k]));
        // (the update is a small part of the parameter: 2^-22 of it is far below the parameter's own rounding)
        asm("div.approx.f32 %0, %1, %2;" : "=f"(share) : "f"(m[k]), "f"(fmaf(root, s2, h.eps)));
        p[k] = fmaf(-a, share, __fmul_rn(p[k], decay));
    }
    uint32_t r[8];
    if (h.seeded && (BITS == 8 || t.ptype == PACER_BF16))
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t i = place<VEC>(base, lane, k);
            r[k] = mix((uint32_t)i ^ key ^ (i >> 32 ? mix((uint32_t)(i >> 32)) : 0u));
        }
    if (t.ptype == PACER_F32) {
        store<VEC>(reinterpret_cast<float *>(t.param), base, lane, n, p);
        if (t.copy) {
            uint32_t o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = __bfloat16_as_ushort(__float2bfloat16_rn(p[k]));
            store16<VEC>(t.copy, base, lane, n, o);
        }
    } else {
        uint32_t o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t b = __float_as_uint(p[k]);
            o[k] = h.seeded && (~b & 0x7f800000u) ? (b + ((r[k] * 0x9E3779B1u) >> 16)) >> 16 : __bfloat16_as_ushort(__float2bfloat16_rn(p[k]));
        }
        store16<VEC>(reinterpret_cast<bf16 *>(t.param), base, lane, n, o);
    }
    if (BITS == 32) {
        store<VEC>(reinterpret_cast<float *>(t.m), base, lane, n, m);
        store<VEC>(reinterpret_cast<float *>(t.v), base, lane, n, v);
        return;
    }
    uint32_t top_m = 0, top_v = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const bool in = VEC || place<VEC>(base, lane, k) < n;
        top_m = max(top_m, in ? __float_as_uint(m[k]) & 0x7fffffffu : 0u);
        top_v = max(top_v, in ? __float_as_uint(v[k]) & 0x7fffffffu : 0u);
    }
    top_m = __reduce_max_sync(0xffffffffu, top_m);
    top_v = __reduce_max_sync(0xffffffffu, top_v);
    float sm, im, sv, iv;
    scale_of(top_m, TOP_M, 1.f / TOP_M, sm, im);
    scale_of(top_v, TOP_V, 1.f / TOP_V, sv, iv);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t dm = h.seeded ? (r[k] & 0xffffu) << 4 : 1u << 19, dv = h.seeded ? (r[k] >> 16) << 4 : 1u << 19;
        const uint32_t bm = __float_as_uint(__fmul_rn(__fmul_rn(fabsf(m[k]), im), DOWN_M)), bv = __float_as_uint(__fmul_rn(__fmul_rn(v[k], iv), DOWN_V));
        cm[k] = min((bm + dm) >> 20, 127u) | (m[k] < 0.f ? 128u : 0u);
        cv[k] = min((bv + dv) >> 20, 255u);
        if (v[k] > 0.f) cv[k] = max(cv[k], 1u);
    }
    store_codes<VEC>(reinterpret_cast<uint8_t *>(t.m), base, lane, n, cm);
    store_codes<VEC>(reinterpret_cast<uint8_t *>(t.v), base, lane, n, cv);
    if (lane == 0) *reinterpret_cast<float2 *>(t.scales + (base >> 8) * 2) = make_float2(sm, sv);
}

template <class T> __device__ __forceinline__ int tensor_of(const T &tab, uint32_t chunk) {
    int lo = 0, hi = tab.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tab.t[mid].first <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}
__device__ __forceinline__ bool aligned(const void *p, int bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

template <int BITS, int CAP>
__global__ void __launch_bounds__(THREADS_W) k_adamw(const __grid_constant__ Table<CAP> tab) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Hyper &h = tab.h;
    float clip = 1.f;
    bool clipped = false;
    if (h.norm) {
        const float norm = __ldcg(h.norm);
        if (!isfinite(norm)) return;       // nothing is changed
        clipped = h.max_norm > 0.f;
        if (clipped) clip = fminf(__fdiv_rn(h.max_norm, __fadd_rn(norm, 1e-6f)), 1.f);
    }
    float a = h.a, s2 = h.s2, decay = h.decay;
    uint32_t step = h.step;
    if (h.step_dev || h.lr_dev) {
        if (h.step_dev) step = (uint32_t)*h.step_dev;
        const double lr = h.lr_dev ? (double)*h.lr_dev : h.lr;
        a = (float)(lr / (1.0 - pow(h.b1d, (double)step)));
        s2 = (float)(1.0 / sqrt(1.0 - pow(h.b2d, (double)step)));
        decay = (float)(1.0 - lr * h.wd);
    }
    const int i = tensor_of(tab, blockIdx.x), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Item t = tab.t[i];
    const uint32_t key = mix(h.seed ^ mix(step ^ mix((uint32_t)(tab.number + i))));
    const bool vec = aligned(t.param, 16) && aligned(t.copy, 16) && aligned(t.grad, 16) && aligned(t.m, BITS == 32 ? 16 : 8) && aligned(t.v, BITS == 32 ? 16 : 8);
    const int64_t start = (int64_t)(blockIdx.x - t.first) * CHUNK + warp * 256;
#pragma unroll 1
    for (int64_t base = start; base < start + CHUNK && base < t.numel; base += PASS) {
        if (vec && base + 256 <= t.numel) update<BITS, true>(t, h, a, s2, decay, clip, clipped, key, base, lane);
        else update<BITS, false>(t, h, a, s2, decay, clip, clipped, key, base, lane);
    }
}

template <int BITS, int CAP> static cudaError_t launch(const pacer_adamw_tensor *tbl, int from, int to, const Hyper &h, cudaStream_t st) {
    Table<CAP> tab;
    tab.h = h;
    tab.number = from;
    tab.n = 0;
    uint64_t chunks = 0;
    for (int i = from; i < to; ++i) {
        const pacer_adamw_tensor &t = tbl[i];
        tab.t[tab.n++] = {t.param, (bf16 *)t.copy, t.grad, t.exp_avg, t.exp_avg_sq, t.scales, t.numel, (uint32_t)chunks, (uint16_t)t.param_type, (uint16_t)t.grad_type};
        chunks += (uint64_t)(t.numel + CHUNK - 1) / CHUNK;
    }
    if (!chunks) return cudaSuccess;
    if (chunks > 0x7fffffffu) return cudaErrorInvalidValue;
    k_adamw<BITS, CAP><<<(unsigned)chunks, THREADS_W, 0, st>>>(tab);
    return cudaGetLastError();
}

cudaError_t adamw(const pacer_adamw_tensor *tbl, int n, const pacer_adamw_cfg &cfg, cudaStream_t st) {
    Hyper h;
    h.b1 = (float)cfg.beta_one; h.c1 = (float)(1.0 - cfg.beta_one); h.b2 = (float)cfg.beta_two; h.c2 = (float)(1.0 - cfg.beta_two);
    h.eps = (float)cfg.eps;
    h.decay = (float)(1.0 - cfg.lr * cfg.weight_decay);
    h.a = (float)(cfg.lr / (1.0 - std::pow(cfg.beta_one, (double)cfg.step)));
    h.s2 = (float)(1.0 / std::sqrt(1.0 - std::pow(cfg.beta_two, (double)cfg.step)));
    h.b1d = cfg.beta_one; h.b2d = cfg.beta_two; h.lr = cfg.lr; h.wd = cfg.weight_decay;
    h.max_norm = (float)cfg.max_norm;
    h.norm = cfg.norm; h.lr_dev = cfg.lr_device; h.step_dev = cfg.step_device;
    h.seeded = cfg.seeded;
    h.seed = (uint32_t)cfg.seed ^ mix((uint32_t)(cfg.seed >> 32));
    h.step = (uint32_t)cfg.step;
    constexpr int MOST = 480;
    for (int i = 0; i < n; i += MOST) {
        const int to = std::min(n, i + MOST), k = to - i;
        cudaError_t e;
        if (cfg.state_bits == 32) e = k <= 16 ? launch<32, 16>(tbl, i, to, h, st) : k <= 96 ? launch<32, 96>(tbl, i, to, h, st) : launch<32, MOST>(tbl, i, to, h, st);
        else e = k <= 16 ? launch<8, 16>(tbl, i, to, h, st) : k <= 96 ? launch<8, 96>(tbl, i, to, h, st) : launch<8, MOST>(tbl, i, to, h, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// ----------------------------------------------------------------------------- 8-bit states as f32

struct StateItem {
    const uint8_t *m, *v;
    const float *scales;
    float *om, *ov;
    int64_t numel;
    uint32_t first, pad;
};
template <int CAP> struct StateTable {
    int32_t n, pad;
    StateItem t[CAP];
};

template <bool VEC> __device__ __forceinline__ void read_states(const StateItem &t, int64_t base, int lane) {
    uint32_t c[8];
    float x[8];
    const float2 s = *reinterpret_cast<const float2 *>(t.scales + (base >> 8) * 2);
    if (t.om) {
        load_codes<VEC>(t.m, base, lane, t.numel, c);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = value_m(c[k], s.x);
        store<VEC>(t.om, base, lane, t.numel, x);
    }
    if (t.ov) {
        load_codes<VEC>(t.v, base, lane, t.numel, c);
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = value_v(c[k], s.y);
        store<VEC>(t.ov, base, lane, t.numel, x);
    }
}
template <int CAP>
__global__ void __launch_bounds__(THREADS_W) k_states(const __grid_constant__ StateTable<CAP> tab) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const StateItem t = tab.t[tensor_of(tab, blockIdx.x)];
    const bool vec = aligned(t.m, 8) && aligned(t.v, 8) && aligned(t.om, 16) && aligned(t.ov, 16);
    const int64_t start = (int64_t)(blockIdx.x - t.first) * CHUNK + warp * 256;
#pragma unroll 1
    for (int64_t base = start; base < start + CHUNK && base < t.numel; base += PASS) {
        if (vec && base + 256 <= t.numel) read_states<true>(t, base, lane);
        else read_states<false>(t, base, lane);
    }
}
template <int CAP>
static cudaError_t launch_states(const pacer_adamw_tensor *tbl, int from, int to, float *const *om, float *const *ov, cudaStream_t st) {
    StateTable<CAP> tab;
    tab.n = 0;
    uint64_t chunks = 0;
    for (int i = from; i < to; ++i) {
        const pacer_adamw_tensor &t = tbl[i];
        tab.t[tab.n++] = {(const uint8_t *)t.exp_avg, (const uint8_t *)t.exp_avg_sq, t.scales, om ? om[i] : nullptr, ov ? ov[i] : nullptr, t.numel, (uint32_t)chunks, 0};
        chunks += (uint64_t)(t.numel + CHUNK - 1) / CHUNK;
    }
    if (!chunks) return cudaSuccess;
    if (chunks > 0x7fffffffu) return cudaErrorInvalidValue;
    k_states<CAP><<<(unsigned)chunks, THREADS_W, 0, st>>>(tab);
    return cudaGetLastError();
}
cudaError_t states(const pacer_adamw_tensor *tbl, int n, float *const *exp_avg, float *const *exp_avg_sq, cudaStream_t st) {
    constexpr int MOST = 480;
    for (int i = 0; i < n; i += MOST) {
        const int to = std::min(n, i + MOST), k = to - i;
        const cudaError_t e = k <= 16 ? launch_states<16>(tbl, i, to, exp_avg, exp_avg_sq, st) : k <= 96 ? launch_states<96>(tbl, i, to, exp_avg, exp_avg_sq, st)
                                                                                             : launch_states<MOST>(tbl, i, to, exp_avg, exp_avg_sq, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// ----------------------------------------------------------------------------- the gradients' norm

struct NormItem {
    const void *p;
    int64_t numel;
    uint32_t first, type;
};
template <int CAP> struct NormTable {
    double *part;                          // of this launch's blocks
    int32_t n;
    uint32_t chunks;
    NormItem t[CAP];
};
constexpr int NORM_CHUNK = 4 * PASS;

// Sums in 64 bits: f32 sums of 10^9 squares would be off in the fifth digit, and the norm scales every gradient.
template <int CAP>
__global__ void __launch_bounds__(THREADS_W) k_norm(const __grid_constant__ NormTable<CAP> tab) {
    __shared__ double red[THREADS_W / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double s0 = 0.0, s1 = 0.0;
    for (uint32_t c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
        const NormItem t = tab.t[tensor_of(tab, c)];
        const bool vec = aligned(t.p, 16);
        const int64_t start = (int64_t)(c - t.first) * NORM_CHUNK + warp * 256;
#pragma unroll 4
        for (int64_t base = start; base < start + NORM_CHUNK && base < t.numel; base += PASS) {
            float x[8];
            if (vec && base + 256 <= t.numel) load<true>(t.p, t.type, base, lane, t.numel, x);
            else load<false>(t.p, t.type, base, lane, t.numel, x);
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                s0 = fma((double)x[k], (double)x[k], s0);
                s1 = fma((double)x[k + 1], (double)x[k + 1], s1);
            }
        }
    }
    s0 += s1;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s0 += __shfl_xor_sync(0xffffffffu, s0, o);
    if (lane == 0) red[warp] = s0;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < THREADS_W / 32; ++w) s0 += red[w];
        tab.part[blockIdx.x] = s0;
    }
}
__global__ void __launch_bounds__(THREADS_W) k_norm_end(const double *part, int n, float *norm) {
    __shared__ double red[THREADS_W / 32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += THREADS_W) s += part[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < THREADS_W / 32; ++w) s += red[w];
    *norm = (float)sqrt(s);
}

size_t norm_scratch_bytes(int n) { return (size_t)((n + NORM_CAP - 1) / NORM_CAP) * NORM_BLOCKS * sizeof(double); }

template <int CAP> static cudaError_t launch_norm(const pacer_gradient *tbl, int from, int to, double *part, int *blocks, cudaStream_t st) {
    NormTable<CAP> tab;
    tab.part = part;
    tab.n = 0;
    uint64_t chunks = 0;
    for (int i = from; i < to; ++i) {
        tab.t[tab.n++] = {tbl[i].grad, tbl[i].numel, (uint32_t)chunks, (uint32_t)tbl[i].type};
        chunks += (uint64_t)(tbl[i].numel + NORM_CHUNK - 1) / NORM_CHUNK;
    }
    *blocks = 0;
    if (!chunks) return cudaSuccess;
    if (chunks > 0x7fffffffu) return cudaErrorInvalidValue;
    tab.chunks = (uint32_t)chunks;
    *blocks = (int)std::min<uint64_t>(chunks, NORM_BLOCKS);
    k_norm<CAP><<<(unsigned)*blocks, THREADS_W, 0, st>>>(tab);
    return cudaGetLastError();
}
cudaError_t grad_norm(const pacer_gradient *tbl, int n, float *norm, double *scratch, cudaStream_t st) {
    int at = 0;
    for (int i = 0; i < n; i += NORM_CAP) {
        const int to = std::min(n, i + NORM_CAP), k = to - i;
        int blocks;
        const cudaError_t e = k <= 32 ? launch_norm<32>(tbl, i, to, scratch + at, &blocks, st) : k <= 256 ? launch_norm<256>(tbl, i, to, scratch + at, &blocks, st)
                                                                                                    : launch_norm<NORM_CAP>(tbl, i, to, scratch + at, &blocks, st);
        if (e != cudaSuccess) return e;
        at += blocks;
    }
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(1);
    c.blockDim = dim3(THREADS_W);
    c.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    c.attrs = attr;
    c.numAttrs = at ? 1 : 0;
    return cudaLaunchKernelEx(&c, k_norm_end, (const double *)scratch, at, norm);
}

}  // namespace ow

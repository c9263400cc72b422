// AdamW over many tensors in one launch, states in 32 or in 8 bits; the global norm of their gradients; 8-bit states as f32.
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// Bound by memory: 28 bytes an element with f32 parameters, gradients and states (50.6 M elements 220 us, 98 % of the copy rate; 131 M with a
// 16-bit gradient and copy 575 us, 97 %), 14 with f32 parameters, 16-bit gradients and 8-bit states (607 M 1445 us, 90 %); with 16-bit
// parameters rounded at random, 10 bytes an element, by its 69 instructions (233 M 530 us, 67 %; with second moments by their roots 646).
// The tensors' table travels in the launch's arguments (no copy to the device, nothing to keep), a block finds its chunk's tensor by bisection.
//
// States in 8 bits, in blocks of 256 elements, the share of a warp (eight elements a lane).  m: sign, 4 exponent and 3 mantissa bits;
// v: 5 exponent and 3 mantissa bits (a second moment spans the square of a first one's range), or its root as 4 exponent and 4 mantissa
// bits (the same range and steps; a correctly rounded root an element more); each times a scale of its block, so that the largest gets the
// largest code.  A code is the upper bits of an f32 number whose exponents were moved down to where the
// code's begin: below them f32 is as evenly spaced as the code, so that coding is one multiplication, an addition and a shift, subnormal values
// included.  What the shift drops decides the rounding: half of it added is rounding to nearest (halves up), 16 random bits added make
// the mean of the code the value.  Rounded to nearest, b2 = 0.999 cannot move a v with steps of an eighth as it should: after 2000 steps its mean
// is 20 % too large, at random it is 0.1 % off.  v above 0 never becomes 0, so that no update is divided by eps alone.
// Products and sums are rounded one by one (no contraction): which of two codes a value gets hangs on its last bit, and is the same wherever
// the formulas are evaluated in f32.
#include "adamw.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "two.cuh"

namespace ow {

using namespace tw;

typedef __nv_bfloat16 bf16;

constexpr int THREADS_W = 256, PASS = 8 * THREADS_W, CHUNK = 4 * PASS;
constexpr int WIDE = 32, SQUARES = 8, ROOTS = 9;           // how states are held: f32; 8-bit codes, v as it is or by its root
// What is held in codes: m, v, the root of v.  The largest code's value, the factors that move exponents to where the code's begin and back, the
// bits of an f32 number below its code.
enum Kind { M, V, R };
template <Kind K> struct Code {
    static constexpr float TOP = K == M ? 480.f : K == V ? 61440.f : 496.f, DOWN = K == V ? 0x1p-111f : 0x1p-120f, UP = K == V ? 0x1p111f : 0x1p120f;
    static constexpr int SHIFT = K == R ? 19 : 20;
};
constexpr float LEAST = 1e-30f;

struct Item {
    void *param;
    bf16 *copy;
    const void *grad;
    void *m, *v;
    float *scales;
    int64_t numel;
    uint32_t first, number;                // chunk; place in the call
};
static_assert(sizeof(Item) == 64, "the table's rows");

struct Hyper {
    float b1, c1, b2, c2, eps, decay, a, s2;
    float max_norm, one;                   // one: 1 (see update)
    uint32_t seed, step;
    const float *norm, *lr_dev;
    const int32_t *step_dev;
    double b1d, b2d, lr, wd;
    int32_t seeded;
};

template <int CAP> struct Table {
    Hyper h;
    int32_t n, pad;
    Item t[CAP];
};

__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {     // an integer hash (constants: C. Wellons, "Prospecting for hash functions", 2018)
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}

// Eight values of a lane: side by side (VEC), or 32 apart, those below n.
template <bool VEC> __device__ __forceinline__ int64_t place(int64_t base, int lane, int k) { return base + (VEC ? lane * 8 + k : lane + 32 * k); }

__device__ __forceinline__ uint4 ld16(const void *p) {              // (read once: kept out of L1)
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <int TYPE> __device__ __forceinline__ float widen(uint32_t h) {
    return TYPE == PACER_BF16 ? __uint_as_float(h << 16) : __half2float(__ushort_as_half((unsigned short)h));
}
// Eight values as they lie in memory.
template <int TYPE> struct Raw { uint4 v[TYPE == PACER_F32 ? 2 : 1]; };
template <bool VEC, int TYPE> __device__ __forceinline__ void fetch(const void *p, int64_t base, int lane, int64_t n, Raw<TYPE> &r) {
    if (VEC) {
        const char *q = reinterpret_cast<const char *>(p) + (base + lane * 8) * (TYPE == PACER_F32 ? 4 : 2);
        r.v[0] = ld16(q);
        if (TYPE == PACER_F32) r.v[TYPE == PACER_F32] = ld16(q + 16);
    } else {
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t i = place<false>(base, lane, k);
            w[k] = i >= n ? 0u : TYPE == PACER_F32 ? reinterpret_cast<const uint32_t *>(p)[i] : reinterpret_cast<const uint16_t *>(p)[i];
        }
        if (TYPE == PACER_F32) {
            r.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
            r.v[TYPE == PACER_F32] = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
            r.v[0] = make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
        }
    }
}
template <int TYPE> __device__ __forceinline__ void widen8(const Raw<TYPE> &r, float (&x)[8]) {
    const uint4 u = r.v[0], z = r.v[TYPE == PACER_F32];
    const uint32_t w[8] = {u.x, u.y, u.z, u.w, z.x, z.y, z.z, z.w};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (TYPE == PACER_F32) x[k] = __uint_as_float(w[k]);
        else if (TYPE == PACER_BF16) x[k] = __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
        else x[k] = widen<TYPE>(k & 1 ? w[k >> 1] >> 16 : w[k >> 1] & 0xffffu);
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
// The upper halves of eight words
template <bool VEC> __device__ __forceinline__ void store16(bf16 *p, int64_t base, int lane, int64_t n, const uint32_t (&h)[8]) {
    uint16_t *q = reinterpret_cast<uint16_t *>(p);
    if (VEC) *reinterpret_cast<uint4 *>(q + base + lane * 8) = make_uint4(__byte_perm(h[0], h[1], 0x7632), __byte_perm(h[2], h[3], 0x7632),
                                                                          __byte_perm(h[4], h[5], 0x7632), __byte_perm(h[6], h[7], 0x7632));
    else
#pragma unroll
        for (int k = 0; k < 8; ++k) { const int64_t i = place<false>(base, lane, k); if (i < n) q[i] = (uint16_t)(h[k] >> 16); }
}
// Eight codes, four to a word
template <bool VEC> __device__ __forceinline__ uint2 load_codes(const uint8_t *q, int64_t base, int lane, int64_t n) {
    uint2 u = make_uint2(0u, 0u);
    if (VEC) asm volatile("ld.global.L1::no_allocate.v2.b32 {%0,%1}, [%2];" : "=r"(u.x), "=r"(u.y) : "l"(q + base + lane * 8));
    else
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t i = place<false>(base, lane, k);
            const uint32_t c = i < n ? q[i] : 0u;
            if (k < 4) u.x |= c << (8 * k);
            else u.y |= c << (8 * k - 32);
        }
    return u;
}
__device__ __forceinline__ uint32_t top_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
__device__ __forceinline__ uint32_t top_bytes(const float *x) {
    return top_bytes(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <bool VEC> __device__ __forceinline__ void store_codes(uint8_t *q, int64_t base, int lane, int64_t n, uint2 u) {
    if (VEC) *reinterpret_cast<uint2 *>(q + base + lane * 8) = u;
    else
#pragma unroll
        for (int k = 0; k < 8; ++k) { const int64_t i = place<false>(base, lane, k); if (i < n) q[i] = (uint8_t)((k < 4 ? u.x : u.y) >> (8 * (k & 3))); }
}
// The largest size of eight; NaN where there is one.
__device__ __forceinline__ float largest(const float (&x)[8]) {
    float a, b;
    asm("{\n\t.reg .f32 a, b, c;\n\tabs.f32 a, %1;\n\tabs.f32 b, %2;\n\tabs.f32 c, %3;\n\tmax.NaN.f32 %0, a, b, c;\n\t}" : "=f"(a) : "f"(x[0]), "f"(x[1]), "f"(x[2]));
    asm("{\n\t.reg .f32 a, b, c;\n\tabs.f32 a, %1;\n\tabs.f32 b, %2;\n\tabs.f32 c, %3;\n\tmax.NaN.f32 %0, a, b, c;\n\t}" : "=f"(b) : "f"(x[3]), "f"(x[4]), "f"(x[5]));
    asm("{\n\t.reg .f32 a, b;\n\tabs.f32 a, %2;\n\tabs.f32 b, %3;\n\tmax.NaN.f32 %0, %1, a, b;\n\t}" : "=f"(a) : "f"(a), "f"(x[6]), "f"(x[7]));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(a) : "f"(a), "f"(b));
    return a;
}

__device__ __forceinline__ void scale2(float (&x)[8], float f) {
    const Two t = two(f, f);
#pragma unroll
    for (int k = 0; k < 8; k += 2) apart(mul2(two(x[k], x[k + 1]), t), x[k], x[k + 1]);
}

// What eight codes stand for.  The move of the exponents and the scale are one factor, unless that would overflow.
template <Kind K> __device__ __forceinline__ void values(uint2 c, float scale, float (&x)[8]) {
    constexpr float MOST = K == V ? 65536.f : 128.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t w = k < 4 ? c.x : c.y;
        if (K == M) x[k] = __uint_as_float((uint32_t)((int32_t)(w << (24 - 8 * (k & 3))) >> 4) & 0x87f00000u);
        else x[k] = __uint_as_float(__byte_perm(w, 0u, (uint32_t)(k & 3) << 8 | 0x4044u) << (Code<K>::SHIFT - 16));
    }
    if (scale < MOST) scale *= Code<K>::UP;
    else scale2(x, Code<K>::UP);
    scale2(x, scale);
}

// The scale of a block from its largest bits (NaN above all, so that a block with one is NaN from then on).
__device__ __forceinline__ void scale_of(uint32_t bits, float top, float one_by_top, float &scale, float &inverse) {
    const float peak = __uint_as_float(bits);
    const bool none = peak <= LEAST;       // too small to be told from 0: codes and scale are 0
    scale = none ? 0.f : __fmul_rn(peak, one_by_top);
    inverse = none ? 0.f : __fdiv_rn(top, peak);
}

struct Step { float a, s2, decay, clip; bool clipped; };

// What a lane reads of its eight elements, of a warp's 256: a block of 8-bit states.
template <int BITS, int PT, int GT> struct In {
    Raw<GT> g;
    Raw<PT> p;
    Raw<PACER_F32> m, v;                   // (32-bit states)
    uint2 cm, cv;
    float2 scale;
};
template <int BITS, int PT, int GT, bool VEC> __device__ __forceinline__ void fetch_all(const Item &t, int64_t base, int lane, In<BITS, PT, GT> &in) {
    fetch<VEC, GT>(t.grad, base, lane, t.numel, in.g);
    fetch<VEC, PT>(t.param, base, lane, t.numel, in.p);
    if (BITS == WIDE) {
        fetch<VEC, PACER_F32>(t.m, base, lane, t.numel, in.m);
        fetch<VEC, PACER_F32>(t.v, base, lane, t.numel, in.v);
    } else {
        in.cm = load_codes<VEC>(reinterpret_cast<const uint8_t *>(t.m), base, lane, t.numel);
        in.cv = load_codes<VEC>(reinterpret_cast<const uint8_t *>(t.v), base, lane, t.numel);
        in.scale = *reinterpret_cast<const float2 *>(t.scales + (base >> 8) * 2);
    }
}

// key: the tensor's.
template <int BITS, int PT, int GT, bool SEEDED, bool VEC>
__device__ __forceinline__ void update(const Item &t, const Hyper &h, const Step &q, uint32_t key, int64_t base, int lane, const In<BITS, PT, GT> &in) {
    constexpr Kind HELD = BITS == ROOTS ? R : V;
    const int64_t n = t.numel;
    float p[8], g[8], m[8], v[8];
    widen8<GT>(in.g, g);
    widen8<PT>(in.p, p);
    if (BITS == WIDE) {
        widen8<PACER_F32>(in.m, m);
        widen8<PACER_F32>(in.v, v);
    } else {
        values<M>(in.cm, in.scale.x, m);
        values<HELD>(in.cv, in.scale.y, v);
        if (BITS == ROOTS)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __fmul_rn(v[k], v[k]);
    }
    if (q.clipped) scale2(g, q.clip);
    const Two b1 = two(h.b1, h.b1), c1 = two(h.c1, h.c1), b2 = two(h.b2, h.b2), c2 = two(h.c2, h.c2);
    // (as a sum of two products of pairs the assembler would make one product and a multiply-add of it: times 1 they stay what they are)
    const Two one = two(h.one, h.one);
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const Two x = two(g[k], g[k + 1]);
        apart(fma2(mul2(two(m[k], m[k + 1]), b1), one, mul2(x, c1)), m[k], m[k + 1]);
        apart(fma2(mul2(two(v[k], v[k + 1]), b2), one, mul2(mul2(x, x), c2)), v[k], v[k + 1]);
        float r0, r1;
        if (BITS == ROOTS) {               // (from here on v is its root)
            r0 = v[k] = __fsqrt_rn(v[k]);
            r1 = v[k + 1] = __fsqrt_rn(v[k + 1]);
        } else {
            asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(v[k]));
            asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(v[k + 1]));
        }
        apart(fma2(two(r0, r1), two(q.s2, q.s2), two(h.eps, h.eps)), r0, r1);
        // (the update is a small part of the parameter: 2^-22 of it is far below the parameter's own rounding)
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(r0));
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(r1));
        const Two share = mul2(two(m[k], m[k + 1]), two(r0, r1));
        apart(fma2(share, two(-q.a, -q.a), mul2(two(p[k], p[k + 1]), two(q.decay, q.decay))), p[k], p[k + 1]);
    }
    uint32_t r[8];
    constexpr bool seeded = SEEDED && (BITS != WIDE || PT == PACER_BF16);
    if (seeded) {
        // (base is a multiple of 256: the number's lowest bits are the lane's)
        const uint32_t x = (uint32_t)base ^ key ^ ((base >> 32) ? mix((uint32_t)(base >> 32)) : 0u) ^ (uint32_t)(VEC ? lane * 8 : lane);
#pragma unroll
        for (int k = 0; k < 8; ++k) r[k] = mix(x ^ (uint32_t)(VEC ? k : 32 * k));
    }
    if (PT == PACER_F32) {
        store<VEC>(reinterpret_cast<float *>(t.param), base, lane, n, p);
        if (t.copy) {
            uint32_t o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(p[k])) << 16;
            store16<VEC>(t.copy, base, lane, n, o);
        }
    } else {
        uint32_t o[8];
        float odd = 0.f;                   // NaN where one of the eight is not finite: their bits are not to be added to
#pragma unroll
        for (int k = 0; k < 8; ++k) odd = fmaf(p[k], 0.f, odd);
        if (seeded && odd == 0.f) {
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = __float_as_uint(p[k]) + ((r[k] * 0x9E3779B1u) >> 16);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t b = __float_as_uint(p[k]);
                o[k] = seeded && (~b & 0x7f800000u) ? b + ((r[k] * 0x9E3779B1u) >> 16) : (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(p[k])) << 16;
            }
        }
        store16<VEC>(reinterpret_cast<bf16 *>(t.param), base, lane, n, o);
    }
    if (BITS == WIDE) {
        store<VEC>(reinterpret_cast<float *>(t.m), base, lane, n, m);
        store<VEC>(reinterpret_cast<float *>(t.v), base, lane, n, v);
        return;
    }
    if (!VEC)
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (place<VEC>(base, lane, k) >= n) m[k] = v[k] = 0.f;
    const uint32_t top_m = __reduce_max_sync(0xffffffffu, __float_as_uint(largest(m))), top_v = __reduce_max_sync(0xffffffffu, __float_as_uint(largest(v)));
    float sm, im, sv, iv, um[8], uv[8];
    scale_of(top_m, Code<M>::TOP, 1.f / Code<M>::TOP, sm, im);
    scale_of(top_v, Code<HELD>::TOP, 1.f / Code<HELD>::TOP, sv, iv);
#pragma unroll
    for (int k = 0; k < 8; ++k) { um[k] = m[k]; uv[k] = v[k]; }
    scale2(um, im); scale2(um, Code<M>::DOWN);
    scale2(uv, iv); scale2(uv, Code<HELD>::DOWN);
    // A code above the last (the largest, where its quotient was rounded up; NaN) or of 0 with v above 0 is rare, and looked for in a block as a whole.
    constexpr int SM = Code<M>::SHIFT, SV = Code<HELD>::SHIFT;
    uint32_t low = __float_as_uint(uv[0]);
#pragma unroll
    for (int k = 1; k < 8; ++k) low = min(low, __float_as_uint(uv[k]));
    const bool plain = VEC && __reduce_min_sync(0xffffffffu, low) >= 1u << SV &&
                       __float_as_uint(__fmul_rn(__fmul_rn(__uint_as_float(top_m), im), Code<M>::DOWN)) <= 127u << SM &&
                       __float_as_uint(__fmul_rn(__fmul_rn(__uint_as_float(top_v), iv), Code<HELD>::DOWN)) <= 255u << SV;
    uint32_t cm[8], cv[8];                 // the codes in the topmost bytes (m's sign has left)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t dm = seeded ? __byte_perm(r[k], 0u, 0x4104) : 1u << 23, dv = seeded ? __byte_perm(r[k], 0u, 0x4324) : 1u << 23;
        cm[k] = (__float_as_uint(um[k]) << (24 - SM)) + dm;
        cv[k] = (__float_as_uint(uv[k]) << (24 - SV)) + dv;
    }
    if (!plain)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t dm = seeded ? (r[k] & 0xffffu) << (SM - 16) : 1u << (SM - 1), dv = seeded ? r[k] >> 16 << (SV - 16) : 1u << (SV - 1);
            cm[k] = min(((__float_as_uint(um[k]) & 0x7fffffffu) + dm) >> SM, 127u) << 24;
            cv[k] = max(min((__float_as_uint(uv[k]) + dv) >> SV, 255u), min(__float_as_uint(v[k]), 1u)) << 24;
        }
    store_codes<VEC>(reinterpret_cast<uint8_t *>(t.m), base, lane, n,
                     make_uint2(top_bytes(cm[0], cm[1], cm[2], cm[3]) | (top_bytes(m) & 0x80808080u), top_bytes(cm[4], cm[5], cm[6], cm[7]) | (top_bytes(m + 4) & 0x80808080u)));
    store_codes<VEC>(reinterpret_cast<uint8_t *>(t.v), base, lane, n, make_uint2(top_bytes(cv[0], cv[1], cv[2], cv[3]), top_bytes(cv[4], cv[5], cv[6], cv[7])));
    if (lane == 0) *reinterpret_cast<float2 *>(t.scales + (base >> 8) * 2) = make_float2(sm, sv);
}
// (a tensor's last elements, and all of one that lies off the 16-byte grid)
template <int BITS, int PT, int GT, bool SEEDED>
__device__ __noinline__ void update_slow(const Item &t, const Hyper &h, const Step &q, uint32_t key, int64_t base, int lane) {
    In<BITS, PT, GT> in;
    fetch_all<BITS, PT, GT, false>(t, base, lane, in);
    update<BITS, PT, GT, SEEDED, false>(t, h, q, key, base, lane, in);
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

template <int BITS, int PT, int GT, bool SEEDED, int CAP>
__global__ void __launch_bounds__(THREADS_W, BITS != WIDE ? 3 : 4) k_adamw(const __grid_constant__ Table<CAP> tab) {
    const Hyper &h = tab.h;
    Step q{h.a, h.s2, h.decay, 1.f, false};
    if (h.norm) {
        const float norm = __ldcg(h.norm);
        if (!isfinite(norm)) return;       // nothing is changed
        q.clipped = h.max_norm > 0.f;
        if (q.clipped) q.clip = fminf(__fdiv_rn(h.max_norm, __fadd_rn(norm, 1e-6f)), 1.f);
    }
    uint32_t step = h.step;
    if (h.step_dev || h.lr_dev) {
        if (h.step_dev) step = (uint32_t)max(*h.step_dev, 1);
        const double lr = h.lr_dev ? (double)*h.lr_dev : h.lr;
        q.a = (float)(lr / (1.0 - pow(h.b1d, (double)step)));
        q.s2 = (float)(1.0 / sqrt(1.0 - pow(h.b2d, (double)step)));
        q.decay = (float)(1.0 - lr * h.wd);
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Item &t = tab.t[tensor_of(tab, blockIdx.x)];
    const uint32_t key = mix(h.seed ^ mix(step ^ mix(t.number)));
    const bool vec = aligned(t.param, 16) && aligned(t.copy, 16) && aligned(t.grad, 16) && aligned(t.m, BITS == WIDE ? 16 : 8) && aligned(t.v, BITS == WIDE ? 16 : 8);
    const int64_t start = (int64_t)(blockIdx.x - t.first) * CHUNK + warp * 256, end = min(start - warp * 256 + CHUNK, t.numel);
    int64_t base = start;
    if (vec && BITS == WIDE) {
#pragma unroll 1
        for (; base + 256 <= end; base += PASS) {
            In<BITS, PT, GT> in;
            fetch_all<BITS, PT, GT, true>(t, base, lane, in);
            update<BITS, PT, GT, SEEDED, true>(t, h, q, key, base, lane, in);
        }
    } else if (vec && base + 256 <= end) { // (the next elements are on their way while these are worked on: codes take ten times the instructions)
        In<BITS, PT, GT> in, next;
        fetch_all<BITS, PT, GT, true>(t, base, lane, in);
#pragma unroll 1
        while (true) {
            const bool more = base + PASS + 256 <= end;
            if (more) fetch_all<BITS, PT, GT, true>(t, base + PASS, lane, next);
            update<BITS, PT, GT, SEEDED, true>(t, h, q, key, base, lane, in);
            base += PASS;
            if (!more) break;
            in = next;
        }
    }
#pragma unroll 1
    for (; base < end; base += PASS) update_slow<BITS, PT, GT, SEEDED>(t, h, q, key, base, lane);
}

// The tensors at[0 .. n).
template <int BITS, int PT, int GT, bool SEEDED, int CAP> static cudaError_t launch(const pacer_adamw_tensor *tbl, const int *at, int n, const Hyper &h, cudaStream_t st) {
    Table<CAP> tab;
    tab.h = h;
    tab.n = n;
    uint64_t chunks = 0;
    for (int i = 0; i < n; ++i) {
        const pacer_adamw_tensor &t = tbl[at[i]];
        tab.t[i] = {t.param, (bf16 *)t.copy, t.grad, t.exp_avg, t.exp_avg_sq, t.scales, t.numel, (uint32_t)chunks, (uint32_t)at[i]};
        chunks += (uint64_t)(t.numel + CHUNK - 1) / CHUNK;
    }
    if (chunks > 0x7fffffffu) return cudaErrorInvalidValue;
    k_adamw<BITS, PT, GT, SEEDED, CAP><<<(unsigned)chunks, THREADS_W, 0, st>>>(tab);
    return cudaGetLastError();
}
constexpr int MOST = 480;                  // tensors a launch: 32 KB of arguments
template <int BITS, int PT, int GT, bool SEEDED> static cudaError_t launch_sized(const pacer_adamw_tensor *tbl, const int *at, int n, const Hyper &h, cudaStream_t st) {
    return n <= 16 ? launch<BITS, PT, GT, SEEDED, 16>(tbl, at, n, h, st) : n <= 224 ? launch<BITS, PT, GT, SEEDED, 224>(tbl, at, n, h, st) : launch<BITS, PT, GT, SEEDED, MOST>(tbl, at, n, h, st);
}
template <int BITS, int PT, int GT> static cudaError_t launch_some(const pacer_adamw_tensor *tbl, const int *at, int n, const Hyper &h, cudaStream_t st) {
    if (h.seeded && (BITS != WIDE || PT == PACER_BF16)) return launch_sized<BITS, PT, GT, BITS != WIDE || PT == PACER_BF16>(tbl, at, n, h, st);
    return launch_sized<BITS, PT, GT, false>(tbl, at, n, h, st);
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
    h.one = 1.f;
    h.norm = cfg.norm; h.lr_dev = cfg.lr_device; h.step_dev = cfg.step_device;
    h.seeded = cfg.seeded;
    h.seed = (uint32_t)cfg.seed ^ mix((uint32_t)(cfg.seed >> 32));
    h.step = (uint32_t)cfg.step;
    typedef cudaError_t (*Fn)(const pacer_adamw_tensor *, const int *, int, const Hyper &, cudaStream_t);
#define TYPES(BITS)                                                                                                                            \
    {launch_some<BITS, PACER_F32, PACER_F32>, launch_some<BITS, PACER_F32, PACER_BF16>, launch_some<BITS, PACER_F32, PACER_F16>,                 \
     launch_some<BITS, PACER_BF16, PACER_F32>, launch_some<BITS, PACER_BF16, PACER_BF16>, launch_some<BITS, PACER_BF16, PACER_F16>}
    static const Fn fn[3][6] = {TYPES(WIDE), TYPES(SQUARES), TYPES(ROOTS)};
#undef TYPES
    const bool coded = cfg.state_bits == 8;
    for (int kind = 0; kind < (coded ? 12 : 6); ++kind) {              // (one launch for each set of types that there is)
        int at[MOST], k = 0;
        const int types = kind % 6, roots = kind / 6;
        for (int i = 0; i <= n; ++i) {
            if (k == MOST || (i == n && k)) {
                const cudaError_t e = fn[coded ? 1 + roots : 0][types](tbl, at, k, h, st);
                if (e != cudaSuccess) return e;
                k = 0;
            }
            if (i < n && tbl[i].numel && tbl[i].param_type == types / 3 && tbl[i].grad_type == types % 3 && (!coded || tbl[i].v_code == roots)) at[k++] = i;
        }
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

template <bool VEC, Kind HELD> __device__ __forceinline__ void read_states(const StateItem &t, int64_t base, int lane) {
    float x[8];
    const float2 s = *reinterpret_cast<const float2 *>(t.scales + (base >> 8) * 2);
    if (t.om) {
        values<M>(load_codes<VEC>(t.m, base, lane, t.numel), s.x, x);
        store<VEC>(t.om, base, lane, t.numel, x);
    }
    if (t.ov) {
        values<HELD>(load_codes<VEC>(t.v, base, lane, t.numel), s.y, x);
        if (HELD == R)
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = __fmul_rn(x[k], x[k]);
        store<VEC>(t.ov, base, lane, t.numel, x);
    }
}
template <int CAP, Kind HELD>
__global__ void __launch_bounds__(THREADS_W) k_states(const __grid_constant__ StateTable<CAP> tab) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const StateItem t = tab.t[tensor_of(tab, blockIdx.x)];
    const bool vec = aligned(t.m, 8) && aligned(t.v, 8) && aligned(t.om, 16) && aligned(t.ov, 16);
    const int64_t start = (int64_t)(blockIdx.x - t.first) * CHUNK + warp * 256;
#pragma unroll 1
    for (int64_t base = start; base < start + CHUNK && base < t.numel; base += PASS) {
        if (vec && base + 256 <= t.numel) read_states<true, HELD>(t, base, lane);
        else read_states<false, HELD>(t, base, lane);
    }
}
// The tensors at[0 .. n).
template <int CAP, Kind HELD>
static cudaError_t launch_states(const pacer_adamw_tensor *tbl, const int *at, int n, float *const *om, float *const *ov, cudaStream_t st) {
    StateTable<CAP> tab;
    tab.n = n;
    uint64_t chunks = 0;
    for (int k = 0; k < n; ++k) {
        const int i = at[k];
        const pacer_adamw_tensor &t = tbl[i];
        tab.t[k] = {(const uint8_t *)t.exp_avg, (const uint8_t *)t.exp_avg_sq, t.scales, om ? om[i] : nullptr, ov ? ov[i] : nullptr, t.numel, (uint32_t)chunks, 0};
        chunks += (uint64_t)(t.numel + CHUNK - 1) / CHUNK;
    }
    if (chunks > 0x7fffffffu) return cudaErrorInvalidValue;
    k_states<CAP, HELD><<<(unsigned)chunks, THREADS_W, 0, st>>>(tab);
    return cudaGetLastError();
}
template <Kind HELD> static cudaError_t states_held(const pacer_adamw_tensor *tbl, int n, int code, float *const *om, float *const *ov, cudaStream_t st) {
    int at[MOST], k = 0;
    for (int i = 0; i <= n; ++i) {
        if (k == MOST || (i == n && k)) {
            const cudaError_t e = k <= 16 ? launch_states<16, HELD>(tbl, at, k, om, ov, st) : k <= 96 ? launch_states<96, HELD>(tbl, at, k, om, ov, st)
                                                                                                 : launch_states<MOST, HELD>(tbl, at, k, om, ov, st);
            if (e != cudaSuccess) return e;
            k = 0;
        }
        if (i < n && tbl[i].numel && tbl[i].v_code == code) at[k++] = i;
    }
    return cudaSuccess;
}
cudaError_t states(const pacer_adamw_tensor *tbl, int n, float *const *exp_avg, float *const *exp_avg_sq, cudaStream_t st) {
    const cudaError_t e = states_held<V>(tbl, n, PACER_V_SQUARE, exp_avg, exp_avg_sq, st);
    return e != cudaSuccess ? e : states_held<R>(tbl, n, PACER_V_ROOT, exp_avg, exp_avg_sq, st);
}

// ----------------------------------------------------------------------------- the gradients' norm

struct NormItem {
    const void *p;
    int64_t numel;
    uint32_t first, type;
};
constexpr int NORM_CHUNK = 4 * PASS;

template <int CAP> struct NormTable {
    double *part;                          // of this launch's blocks
    int32_t n;
    uint32_t chunks;
    NormItem t[CAP];
};
// |x| in 64 bits by moving its fields: a conversion has a quarter of the rate, which 16-bit gradients at the memory's rate would need in full.
// What is below f32's normal numbers, 0 among it, becomes some number below 2^-126, infinities and NaN some number from 2^128 on, so that
// the norm as f32 is infinite; a norm below 2^-100 is 0.
__device__ __forceinline__ double magnitude(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return __hiloint2double((int)((b >> 3) + (896u << 20)), (int)(b << 29));
}
template <int TYPE> __device__ __forceinline__ void squares(const Raw<TYPE> &r, double &s0, double &s1) {
    float x[8];
    widen8<TYPE>(r, x);
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        const double a = magnitude(x[k]), c = magnitude(x[k + 1]);
        s0 = fma(a, a, s0);
        s1 = fma(c, c, s1);
    }
}
// A warp's part of a chunk; whole ones with all loads under way at once.
template <int TYPE> __device__ __forceinline__ void chunk_squares(const NormItem &t, int64_t base, int64_t end, int lane, double &s0, double &s1) {
    if (aligned(t.p, 16) && base + NORM_CHUNK - PASS + 256 <= end) {
        Raw<TYPE> r[NORM_CHUNK / PASS];
#pragma unroll
        for (int i = 0; i < NORM_CHUNK / PASS; ++i) fetch<true, TYPE>(t.p, base + i * PASS, lane, t.numel, r[i]);
#pragma unroll
        for (int i = 0; i < NORM_CHUNK / PASS; ++i) squares<TYPE>(r[i], s0, s1);
        return;
    }
#pragma unroll 1
    for (; base < end; base += PASS) {
        Raw<TYPE> r;
        fetch<false, TYPE>(t.p, base, lane, t.numel, r);
        squares<TYPE>(r, s0, s1);
    }
}

// Sums in 64 bits: f32 sums of 10^9 squares would be off in the fifth digit, and the norm scales every gradient.
template <int CAP>
__global__ void __launch_bounds__(THREADS_W) k_norm(const __grid_constant__ NormTable<CAP> tab) {
    __shared__ double red[THREADS_W / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    double s0 = 0.0, s1 = 0.0;
    for (uint32_t c = blockIdx.x; c < tab.chunks; c += gridDim.x) {
        const NormItem t = tab.t[tensor_of(tab, c)];
        const int64_t from = (int64_t)(c - t.first) * NORM_CHUNK, end = min(from + NORM_CHUNK, t.numel);
        if (t.type == PACER_F32) chunk_squares<PACER_F32>(t, from + warp * 256, end, lane, s0, s1);
        else if (t.type == PACER_BF16) chunk_squares<PACER_BF16>(t, from + warp * 256, end, lane, s0, s1);
        else chunk_squares<PACER_F16>(t, from + warp * 256, end, lane, s0, s1);
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
    s = sqrt(s);
    *norm = s < 0x1p-100 ? 0.f : (float)s;      // (what zeros add up to)
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

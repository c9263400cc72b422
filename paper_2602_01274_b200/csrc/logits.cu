// Operators on rows of logits: log probabilities of given tokens with entropy and the best alternatives, distillation from a
// teacher's top logits, and their gradients.
//
// All are bound by HBM: a row is read once (and its gradient written once).  A row belongs to a cluster of C blocks, each with a
// share of its 16-byte vectors, so that one row can have the loads of up to eight SMs in flight; with many rows C is 1.  What needs a
// row twice (its best elements, its gradient) reads it again out of L2.
// Softmax sums are held as (m, S), S = sum 2^(z scale - m): the reference m is raised only when a logit lies more than 2^SLACK above
// it (S stays below vocab * 2^SLACK), so that the common path has no rescaling and an exponent is one fused multiply-add.  That is
// right to the exponent's own rounding whatever the logits of a row have in common, and m and log2 S stay apart for what is computed
// from them: their sum would be rounded at the logits' size (0.06 at 1e6), and a log probability with it.  Rows whose largest logit is
// beyond HUGE_M (a row masked with the type's lowest value, say) are summed again, with differences taken first.
#include "logits.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "../../include/pacer.h"

namespace lg {

constexpr int THREADS = 256, WARPS = THREADS / 32, MAX_C = 8;
constexpr int UNROLL = 4;                  // 16-byte vectors of a thread in a batch
constexpr int BATCH = UNROLL * THREADS;    // vectors of a block's batch
constexpr int PER_SM = 5;                  // blocks on an SM
constexpr int CAND = 512;                  // candidates for the alternatives that a block collects at most
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
// 1 / LOG2E as it stands in f32, in two parts: from exponents back to the logits' units at one rounding
constexpr float UNIT_HI = (float)(1.0 / (double)LOG2E), UNIT_LO = (float)(1.0 / (double)LOG2E - (double)UNIT_HI);
constexpr float LOWEST = -3.402823466e38f, SLACK = 16.f;
constexpr float FAR = -1000.f;             // exponents are cut here: 2^FAR is 0, and 0 * FAR too
constexpr float HUGE_M = 1e8f;
constexpr float LSE_EXACT = 1024.f;        // half a step of an f32 log-sum-exp below it is at most 3e-5 of a probability; larger ones are taken anew

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {      // NaN if either is
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// ------------------------------------------------------------------ rows of 16-byte vectors

template <class T> struct Vec;
template <> struct Vec<float> {
    static constexpr int E = 4, KEY_LOW = 0;             // KEY_LOW: low bits of a value as f32 that are always 0
    static constexpr uint32_t NONE = 0xff800000u;        // -inf
    __device__ static float max(const uint4 *v, int n) {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < n; ++i)
            m = fmaxf(fmaxf(fmaxf(m, __uint_as_float(v[i].x)), fmaxf(__uint_as_float(v[i].y), __uint_as_float(v[i].z))), __uint_as_float(v[i].w));
        return m;
    }
    __device__ static void unpack(const uint4 &v, float (&f)[4]) {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    __device__ static uint4 pack(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    // The first reference of a sum is START: what lies far below it (a mask of -1e20, say) adds nothing, as it would add nothing to
    // any row that is not huge().  Where sums of 2^t t are wanted, what lies below LOW counts as LOW, which has 2^t = 0 over START
    // already: 0 * -inf would be NaN.  LEAST: a row whose largest logit is not above it is summed apart (START or LOW could count).
    static constexpr float LOW = -1e30f, START = -HUGE_M, LEAST = -HUGE_M;
    __device__ static void lift(uint4 &v) {                             // (NaN stays)
        v.x = __float_as_uint(max_nan(__uint_as_float(v.x), LOW)); v.y = __float_as_uint(max_nan(__uint_as_float(v.y), LOW));
        v.z = __float_as_uint(max_nan(__uint_as_float(v.z), LOW)); v.w = __float_as_uint(max_nan(__uint_as_float(v.w), LOW));
    }
    __device__ static void hide(uint4 &v, uint32_t w) {                 // -inf in place of the elements whose bit is set
        if (w & 1) v.x = NONE;
        if (w & 2) v.y = NONE;
        if (w & 4) v.z = NONE;
        if (w & 8) v.w = NONE;
    }
    __device__ static float to(float x) { return x; }
    __device__ static float from(float x) { return x; }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int E = 8, KEY_LOW = 16;
    static constexpr uint32_t NONE = 0xff80ff80u;
    __device__ static float max(const uint4 *v, int n) {                // (packed: two values an instruction; NaN is passed over)
        const auto h = [](const uint32_t &u) { return *reinterpret_cast<const __nv_bfloat162 *>(&u); };
        __nv_bfloat162 m = h(v[0].x);
#pragma unroll
        for (int i = 0; i < n; ++i) m = __hmax2(__hmax2(m, h(v[i].x)), __hmax2(__hmax2(h(v[i].y), h(v[i].z)), h(v[i].w)));
        return fmaxf(fmaxf(__low2float(m), __high2float(m)), -INFINITY);
    }
    __device__ static void two(uint32_t u, float &a, float &b) { a = __uint_as_float(u << 16); b = __uint_as_float(u & 0xffff0000u); }
    __device__ static void unpack(const uint4 &v, float (&f)[8]) {
        two(v.x, f[0], f[1]); two(v.y, f[2], f[3]); two(v.z, f[4], f[5]); two(v.w, f[6], f[7]);
    }
    __device__ static uint32_t one(float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    __device__ static uint4 pack(const float (&f)[8]) { return make_uint4(one(f[0], f[1]), one(f[2], f[3]), one(f[4], f[5]), one(f[6], f[7])); }
    static constexpr uint32_t LOW = 0xf14af14au;          // -1e30
    static constexpr float START = -HUGE_M, LEAST = -HUGE_M;
    __device__ static uint32_t lift(uint32_t u) {
        const uint32_t l = LOW;
        const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&u), *reinterpret_cast<const __nv_bfloat162 *>(&l));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
    __device__ static void lift(uint4 &v) { v.x = lift(v.x); v.y = lift(v.y); v.z = lift(v.z); v.w = lift(v.w); }
    __device__ static void hide(uint4 &v, uint32_t w) {
        uint32_t *u = &v.x;
#pragma unroll
        for (int i = 0; i < 4; ++i, w >>= 2) {
            if (w & 1) u[i] = (u[i] & 0xffff0000u) | (NONE & 0xffffu);
            if (w & 2) u[i] = (u[i] & 0xffffu) | (NONE & 0xffff0000u);
        }
    }
    __device__ static float to(__nv_bfloat16 x) { return __bfloat162float(x); }
    __device__ static __nv_bfloat16 from(float x) { return __float2bfloat16_rn(x); }
};
template <> struct Vec<__half> {
    static constexpr int E = 8, KEY_LOW = 13;
    static constexpr uint32_t NONE = 0xfc00fc00u;
    __device__ static float max(const uint4 *v, int n) {
        const auto h = [](const uint32_t &u) { return *reinterpret_cast<const __half2 *>(&u); };
        __half2 m = h(v[0].x);
#pragma unroll
        for (int i = 0; i < n; ++i) m = __hmax2(__hmax2(m, h(v[i].x)), __hmax2(__hmax2(h(v[i].y), h(v[i].z)), h(v[i].w)));
        return fmaxf(fmaxf(__low2float(m), __high2float(m)), -INFINITY);
    }
    __device__ static void two(uint32_t u, float &a, float &b) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u));
        a = f.x; b = f.y;
    }
    __device__ static void unpack(const uint4 &v, float (&f)[8]) {
        two(v.x, f[0], f[1]); two(v.y, f[2], f[3]); two(v.z, f[4], f[5]); two(v.w, f[6], f[7]);
    }
    __device__ static uint32_t one(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    __device__ static uint4 pack(const float (&f)[8]) { return make_uint4(one(f[0], f[1]), one(f[2], f[3]), one(f[4], f[5]), one(f[6], f[7])); }
    static constexpr uint32_t LOW = 0xfbfffbffu;          // the lowest finite value, -65504
    static constexpr float START = -60000.f, LEAST = -30000.f;
    __device__ static uint32_t lift(uint32_t u) {
        const uint32_t l = LOW;
        const __half2 r = __hmax2_nan(*reinterpret_cast<const __half2 *>(&u), *reinterpret_cast<const __half2 *>(&l));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
    __device__ static void lift(uint4 &v) { v.x = lift(v.x); v.y = lift(v.y); v.z = lift(v.z); v.w = lift(v.w); }
    __device__ static void hide(uint4 &v, uint32_t w) {
        uint32_t *u = &v.x;
#pragma unroll
        for (int i = 0; i < 4; ++i, w >>= 2) {
            if (w & 1) u[i] = (u[i] & 0xffff0000u) | (NONE & 0xffffu);
            if (w & 2) u[i] = (u[i] & 0xffffu) | (NONE & 0xffff0000u);
        }
    }
    __device__ static float to(__half x) { return __half2float(x); }
    __device__ static __half from(float x) { return __float2half_rn(x); }
};

// The vectors of a row: vector j holds the elements j * E - off .. j * E - off + E - 1 that lie in [0, vocab) (the row starts
// `off` elements past a 16-byte boundary, so the first and last vector may be partial).  `lo`..`hi`: this block's whole vectors.
template <class T>
struct Share {
    static constexpr int E = Vec<T>::E;
    const T *row;
    int32_t vocab, off, lo, hi, first, last;             // first / last: a partial vector of this block, or -1

    // (2^shift blocks; a division of 64-bit numbers here would cost as much as a quarter of a thread's work on a row)
    __device__ Share(const T *row_, int vocab_, int rank, int shift) : row(row_), vocab(vocab_) {
        off = (int)(((uintptr_t)row & 15) / sizeof(T));
        const uint32_t ends = (uint32_t)off + (uint32_t)vocab, nv = (ends + E - 1) / E;
        lo = (int)(nv * (uint32_t)rank >> shift);
        hi = (int)(nv * (uint32_t)(rank + 1) >> shift);
        first = last = -1;
        if (lo < hi && lo == 0 && (off || vocab < E)) first = lo++;
        if (lo < hi && hi == (int)nv && ends % E) last = --hi;
    }
    __device__ const uint4 *vecs() const { return reinterpret_cast<const uint4 *>(row - off); }
    __device__ int begin(int j) const { return max(j * E - off, 0); }
    __device__ int end(int j) const { return min((j + 1) * E - off, vocab); }
    // Elements of the partial vectors, one a thread: its number, or -1.
    __device__ int edge(int tid) const {
        const int j = tid < E ? first : tid < 2 * E ? last : -1, i = j >= 0 ? begin(j) + tid % E : 0;
        return j >= 0 && i < end(j) ? i : -1;
    }
    // elements of the block: [from, to)
    __device__ int from() const { return first >= 0 ? begin(first) : begin(lo); }
    __device__ int to() const { return last >= 0 ? end(last) : hi > lo ? end(hi - 1) : first >= 0 ? end(first) : from(); }
};

__device__ __forceinline__ uint4 ld_row(const uint4 *p) {        // (not the read-only path: a gradient may go where its logits were)
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
// A thread's vectors lo + tid, lo + tid + THREADS, ..: batch(vectors, first number) for UNROLL at a time, single(vector, number) for
// the last ones, which are loaded together too (one after the other they cost a memory latency each: 263 against 246 us for the
// loss and gradient of 997 rows of 151 936 f32 with a tail).
template <class T, class F, class G>
__device__ __forceinline__ void each_vec(const Share<T> &sh, F batch, G single) {
    int j = sh.lo + threadIdx.x;
    for (; j + (UNROLL - 1) * THREADS < sh.hi; j += UNROLL * THREADS) {
        uint4 v[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) v[u] = ld_row(sh.vecs() + j + u * THREADS);
        batch(v, j);
    }
    uint4 v[UNROLL - 1][1];
#pragma unroll
    for (int u = 0; u < UNROLL - 1; ++u)
        if (j + u * THREADS < sh.hi) v[u][0] = ld_row(sh.vecs() + j + u * THREADS);
#pragma unroll
    for (int u = 0; u < UNROLL - 1; ++u)
        if (j + u * THREADS < sh.hi) single(v[u], j + u * THREADS);
}

// The same from the last vectors to the first: what a pass before it read last is still in L1 (2048 rows of 32 000 bf16, loss and
// gradient: 54.2 against 54.9 us).
template <class T, class F, class G>
__device__ __forceinline__ void each_vec_back(const Share<T> &sh, F batch, G single) {
    const int n = sh.hi - sh.lo - (int)threadIdx.x;                     // (the thread's vectors lie within the next n)
    int j = sh.lo + threadIdx.x + max(0, (n + THREADS - 1) / BATCH) * BATCH;
    uint4 v[UNROLL - 1][1];
#pragma unroll
    for (int u = 0; u < UNROLL - 1; ++u)
        if (j + u * THREADS < sh.hi) v[u][0] = ld_row(sh.vecs() + j + u * THREADS);
#pragma unroll
    for (int u = 0; u < UNROLL - 1; ++u)
        if (j + u * THREADS < sh.hi) single(v[u], j + u * THREADS);
    for (j -= BATCH; j >= sh.lo; j -= BATCH) {
        uint4 w[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) w[u] = ld_row(sh.vecs() + j + u * THREADS);
        batch(w, j);
    }
}

// ------------------------------------------------------------------ softmax sums

// Two fp32 values in one register pair: one instruction works on both.
typedef unsigned long long f2;
__device__ __forceinline__ f2 two(float a, float b) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void apart(f2 v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// S = sum 2^t, S2 = sum 2^t t with t = (z - ref) scale - m.  A logit of -inf adds nothing; NaN and +inf make the sums NaN.
struct Sums {
    float ref = 0.f, m = 0.f, S = 0.f, S2 = 0.f;
    __device__ float exponent(float z, float scale) const { return fmaf(z - ref, scale, -m); }
    // log p of a logit from its exponent (whose range a finite logit far below the others may leave where its log p does not).  At most 0:
    // m is a rounded product, so the only token of a row has 2^t a rounding off 1, and log S one off t
    __device__ float log_p(float z, float scale, float inv_temp, float log2S) const {
        const float e = exponent(z, scale) - log2S;
        return e == -INFINITY ? (z - ref) * inv_temp - (m + log2S) * LN2 : e > 0.f ? 0.f : e * LN2;
    }
};

// A thread's sums while it reads its vectors: even and odd elements apart.
template <class T, bool ENTROPY>
struct PairSums {
    float m = Vec<T>::START;
    f2 S = 0, S2 = 0;
    __device__ void reach(float top) {                                   // the largest exponent (scaled logit) that comes next
        if (top > m + SLACK) {
            const float d = fmaxf(m - top, FAR), r = ex2(d);
            if (ENTROPY) S2 = mul2(two(r, r), fma2(S, two(d, d), S2));
            S = mul2(two(r, r), S);
            m = top;
        }
    }
    // -inf has 2^t = 0, but 0 * t is NaN: a thread whose sum of products turns NaN takes the vectors again lifted, and all that follow
    bool lifted = false;
    template <int N>
    __device__ void add(uint4 (&v)[N], float scale) {
        if (!ENTROPY) { sum<N, false>(v, scale); return; }
        if (!lifted) {
            const f2 S0 = S, P0 = S2;
            sum<N, false>(v, scale);
            float a, b;
            apart(S2, a, b);
            if (!isnan(a + b)) return;
            S = S0; S2 = P0;
            lifted = true;
        }
        sum<N, true>(v, scale);
    }
    template <int N, bool LIFT>
    __device__ void sum(const uint4 (&v)[N], float scale) {
        constexpr int E = Vec<T>::E;
        const f2 c = two(scale, scale), nm = two(-m, -m);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float f[E];
            uint4 w = v[u];
            if (LIFT) Vec<T>::lift(w);
            Vec<T>::unpack(w, f);
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const f2 t = fma2(two(f[e], f[e + 1]), c, nm);
                float t0, t1;
                apart(t, t0, t1);
                const f2 x = two(ex2(t0), ex2(t1));
                S = add2(S, x);
                if (ENTROPY) S2 = fma2(x, t, S2);
            }
        }
    }
    __device__ void add(float z, float scale) {
        reach(z * scale);
        const float t = max_nan(fmaf(z, scale, -m), FAR), x = ex2(t);
        S = add2(S, two(x, 0.f));
        if (ENTROPY) S2 = fma2(two(x, 0.f), two(t, 0.f), S2);
    }
};

__device__ __forceinline__ void barrier_cluster() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer(const void *smem, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(smem)), "r"(rank));
    return r;
}
__device__ __forceinline__ void st_peer(uint32_t at, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory"); }
__device__ __forceinline__ void st_peer64(uint32_t at, uint64_t v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(v) : "memory"); }

// The sums of N = 2^i lanes (lane, lane ^ 1, ..), each with its own reference, over the reference m of them all.
template <int N>
__device__ __forceinline__ void join_lanes(float &m, float &S, float &S2, float scale_m, int n = N) {
    const float top = warp_max(m), d = fmaxf((m - top) * scale_m, FAR), r = ex2(d);
    S2 = r * fmaf(S, d, S2);
    S *= r;
    m = top;
#pragma unroll
    for (int o = 1; o < N; o <<= 1)
        if (o < n) { S += __shfl_xor_sync(~0u, S, o); S2 += __shfl_xor_sync(~0u, S2, o); }
}

struct SumSlots {
    float4 warp[WARPS], block[MAX_C];
};
// The sums of the block's threads in all of them, in a fixed order.  scale_m: from differences of m to exponents.
__device__ __forceinline__ void block_sums(float &m, float &S, float &S2, SumSlots &sl, float scale_m) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    join_lanes<32>(m, S, S2, scale_m);
    if (lane == 0) sl.warp[warp] = make_float4(m, S, S2, 0.f);
    __syncthreads();
    const float4 w = sl.warp[lane % WARPS];
    m = w.x; S = w.y; S2 = w.z;
    join_lanes<WARPS>(m, S, S2, scale_m);
}

// The sums of a whole row by one block, differences of logits taken first: for rows whose scaled logits or log-sum-exp say too
// little (HUGE_M, LSE_EXACT).  skip(i): tokens to leave out.
template <class T, class Skip>
__device__ __noinline__ Sums whole_row(const T *z, int vocab, float scale, SumSlots &sl, Skip skip) {
    constexpr int E = Vec<T>::E;
    const Share<T> sh(z, vocab, 0, 0);
    float m = LOWEST, S = 0.f, S2 = 0.f;                                 // (m unscaled)
    auto add = [&](float x, int i) {
        if (skip(i)) return;
        if (x > m) {
            const float d = fmaxf((m - x) * scale, FAR), r = ex2(d);
            S2 = r * fmaf(S, d, S2);
            S *= r;
            m = x;
        }
        const float t = max_nan((x - m) * scale, FAR), p = ex2(t);
        S += p;
        S2 = fmaf(p, t, S2);
    };
    auto vec = [&](const uint4 &v, int j) {
        float f[E];
        Vec<T>::unpack(v, f);
#pragma unroll
        for (int e = 0; e < E; ++e) add(f[e], j * E - sh.off + e);
    };
#pragma unroll 4
    for (int j = sh.lo + threadIdx.x; j < sh.hi; j += THREADS) vec(ld_row(sh.vecs() + j), j);
    if (const int i = sh.edge(threadIdx.x); i >= 0) add(Vec<T>::to(z[i]), i);
    __syncthreads();                                                     // (the slots may still be read)
    block_sums(m, S, S2, sl, scale);
    Sums s;
    s.ref = m; s.m = 0.f; s.S = S; s.S2 = S2;
    return s;
}

template <class T>
__device__ __forceinline__ bool huge(float m, float scale) { return !(m < HUGE_M && m > Vec<T>::LEAST * fminf(1.f, scale)); }

// The row's sums in every thread of every block of the cluster, in a fixed order; the cluster (or block) is in step after it.
template <class T, class Skip>
__device__ __forceinline__ Sums row_sums(float m, f2 S_, f2 S2_, const Share<T> &sh, SumSlots &sl, int rank, int C, float scale, Skip skip) {
    float S, S2, b;
    apart(S_, S, b); S += b;
    apart(S2_, S2, b); S2 += b;
    __syncwarp();
    if (C > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");      // (the peers run: see the kernels' first lines)
    block_sums(m, S, S2, sl, 1.f);
    if (C > 1) {
        if ((int)threadIdx.x < C) {
            const uint32_t at = peer(&sl.block[rank], threadIdx.x);
            st_peer(at, m); st_peer(at + 4, S); st_peer(at + 8, S2);
        }
        barrier_cluster();
        const float4 w = sl.block[threadIdx.x & (C - 1)];
        m = w.x; S = w.y; S2 = w.z;
        join_lanes<MAX_C>(m, S, S2, 1.f, C);
    }
    if (huge<T>(m, scale)) {                                             // (in all blocks of the cluster alike)
        const Sums s = whole_row<T>(sh.row, sh.vocab, scale, sl, skip);
        if (C > 1) barrier_cluster();                                    // the gradient may go where the logits are
        return s;
    }
    Sums s;
    s.m = m; s.S = S; s.S2 = S2;
    return s;
}

// ------------------------------------------------------------------ alternatives

// Order of the alternatives: larger logit first, then the lower index; NaN last.  A logit as an integer of that order (0: NaN):
__device__ __forceinline__ uint32_t order_key(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);                       // -0 and 0 are equal
    return isnan(z) ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t k) { return __uint_as_float(k == 0u ? 0x7fffffffu : (k & 0x80000000u) ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ uint64_t pair_key(float z, int idx) { return ((uint64_t)order_key(z) << 32) | (uint32_t)~idx; }

constexpr int AGAIN = 512;                 // batches that are looked at again at most

struct TopSlots {
    union {
        struct { uint32_t key[THREADS]; int32_t vec[THREADS]; int32_t equal[THREADS]; };     // while the bound is looked for
        uint64_t cand[CAND];
    };
    uint64_t best[MAX_TOP];
    uint16_t again[AGAIN];
    int32_t n_again, n_cand, bound_idx, ties;
    uint32_t bound;
    int32_t count[WARPS];
};

__device__ __forceinline__ int warp_count(int v) { return __reduce_add_sync(~0u, v); }

// The `top` best elements of the block's share, in order, to best[] (with fewer elements: all, the rest 0).  Thread tid has read the
// whole vectors lo + tid, lo + tid + THREADS, .., and left the largest value of each of its `runs` runs of `run` of them in seg[][tid].
// The top-th best of the 256 per-thread maxima bounds the top-th best element from below; only runs that reach the bound are
// read again, out of L2 (2048 rows of 32 003 bf16, top 64: 79 runs of four vectors of 1000, 82 candidates).
template <class T>
__device__ void block_top(const Share<T> &sh, const float (*seg)[THREADS], int runs, int run, bool has_nan, int top, TopSlots &s) {
    constexpr int E = Vec<T>::E, N = THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nv = sh.hi - sh.lo, RUN = run * THREADS;
    const uint4 *buf = sh.vecs() + sh.lo;
    const bool mine = tid < nv;
    float bv = -INFINITY;
    int bseg = 0;
    for (int g = 0; g < runs; ++g) {
        const float v = seg[g][tid];
        if (v > bv) { bv = v; bseg = g; }
    }
    // (a maximum that ignores NaN says nothing certain about a thread that saw only -inf: it then counts as lowest)
    const uint32_t key = !mine || (has_nan && bv == -INFINITY) ? 0u : order_key(bv);
    s.key[tid] = key;
    if (tid == 0) { s.n_again = s.n_cand = s.ties = 0; s.bound = 0; s.bound_idx = INT32_MAX; }
    __syncthreads();
    if (warp == 0 && min(nv, THREADS) >= top) {
        uint32_t k[N], hi = 0, lo = ~0u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            k[i] = s.key[i * 32 + lane];
            if (i * 32 + lane < nv) { hi = max(hi, k[i]); lo = min(lo, k[i]); }
        }
        hi = __reduce_max_sync(~0u, hi); lo = __reduce_min_sync(~0u, lo);
        // a bound that at least `top` maxima reach, and few more unless they are equal: bit by bit below the bits they share
        const int first = hi == lo ? 0 : 32 - __clz(hi ^ lo);
        uint32_t bound = first == 32 ? 0u : hi >> first << first;
        for (int b = first - 1; b >= Vec<T>::KEY_LOW; --b) {
            const uint32_t trial = bound | (1u << b);
            int n = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) n += k[i] >= trial;
            n = warp_count(n);
            if (n >= top) {
                bound = trial;
                if (n <= top + 4 + top / 8) break;
            }
        }
        if (hi == lo) bound = hi;
        else if (bound && !(bound & 0x80000000u)) bound |= (1u << Vec<T>::KEY_LOW) - 1;      // a negative value's low bits are 1
        int above = 0, equal = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) { above += k[i] > bound; equal += k[i] == bound; }
        above = warp_count(above); equal = warp_count(equal);
        if (above + equal < top) bound = 0;                            // (cannot be)
        if (lane == 0) {
            s.bound = bound;
            s.ties = bound && above + equal > top + 32 ? top - above : 0;
        }
    }
    __syncthreads();
    const uint32_t bound = s.bound;
    if (s.ties > 0) {                                                  // of many equal maxima only the first vectors are needed
        int at = INT32_MAX, equal = 0;
        if (key == bound && mine)
            for (int i = bseg * RUN + tid; i < min((bseg + 1) * RUN, nv) && at == INT32_MAX; i += THREADS)
                if (const uint4 v = ld_row(buf + i); Vec<T>::max(&v, 1) == bv) {
                    float x[E];
                    Vec<T>::unpack(v, x);
                    at = sh.lo + i;
#pragma unroll
                    for (int e = 0; e < E; ++e) equal += x[e] == bv;
                }
        s.vec[tid] = at; s.equal[tid] = equal;
        __syncthreads();
        if (warp == 0) {
            int v[N], c[N], lim = 0;                                   // least vector number with `ties` such elements up to it
#pragma unroll
            for (int i = 0; i < N; ++i) { v[i] = s.vec[i * 32 + lane]; c[i] = s.equal[i * 32 + lane]; }
            for (int b = 31 - __clz(sh.hi); b >= 0; --b) {
                const int trial = lim | (1 << b);
                int n = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) n += v[i] < trial ? c[i] : 0;
                if (warp_count(n) < s.ties) lim = trial;
            }
            if (lane == 0) s.bound_idx = sh.end(min(lim, sh.hi - 1)) - 1;
        }
        __syncthreads();
    }
    const int bound_idx = s.bound_idx;
    const uint64_t least = ((uint64_t)bound << 32) | (uint32_t)~bound_idx;
    const float least_value = bound > order_key(-INFINITY) ? order_value(bound) : -INFINITY;
    auto test = [&](float z, int i) {
        const uint64_t k = pair_key(z, i);
        if (k >= least) {
            const int at = atomicAdd(&s.n_cand, 1);
            if (at < CAND) s.cand[at] = k;
        }
    };
    for (int g = 0; g < runs; ++g) {
        const int i0 = g * RUN + tid;
        const float v = seg[g][tid];
        const bool hit = i0 < nv && (has_nan || v > least_value || (v == least_value && sh.begin(sh.lo + i0) <= bound_idx));
        const uint32_t all = __ballot_sync(~0u, hit);
        if (!all) continue;
        int at = 0;
        if (lane == 0) at = atomicAdd(&s.n_again, __popc(all));
        at = __shfl_sync(~0u, at, 0) + __popc(all & ((1u << lane) - 1));
        if (hit && at < AGAIN) s.again[at] = (uint16_t)(g * THREADS + tid);
    }
    __syncthreads();
    const int again = min(s.n_again, AGAIN);
    for (int w0 = tid; w0 < again * UNROLL; w0 += 2 * THREADS)         // (two vectors on their way)
        for (int p = 0; p < run; p += UNROLL) {
            uint4 v[2];
            int at[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int w = w0 + h * THREADS, f = w < again * UNROLL ? s.again[w / UNROLL] : 0;
                const int i = f / THREADS * RUN + f % THREADS + (p + w % UNROLL) * THREADS;
                at[h] = w < again * UNROLL && i < nv ? i : -1;
                if (at[h] >= 0) v[h] = ld_row(buf + i);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (at[h] < 0 || (!has_nan && Vec<T>::max(v + h, 1) < least_value)) continue;
                float x[E];
                Vec<T>::unpack(v[h], x);
                uint32_t hits = 0;                                     // (one or two of a vector: a branch for each element would cost
#pragma unroll                                                          // the warp eight of them)
                for (int e = 0; e < E; ++e) hits |= has_nan || x[e] >= least_value ? 1u << e : 0u;
                for (; hits; hits &= hits - 1) {
                    const int e = __ffs(hits) - 1;
                    float z = x[0];
#pragma unroll
                    for (int q = 1; q < E; ++q) z = q == e ? x[q] : z;
                    test(z, sh.begin(sh.lo + at[h]) + e);
                }
            }
        }
    if (const int i = sh.edge(tid); i >= 0) test(Vec<T>::to(sh.row[i]), i);
    __syncthreads();
    int n = s.n_cand;
    if (n > CAND || s.n_again > AGAIN) {                                      // (many elements of few threads, or NaN): bit by bit
        uint64_t bar = 0;
        __syncthreads();
        for (int b = 63; b >= 0; --b) {
            const uint64_t trial = bar | (1ull << b);
            int c = 0;
            for (int i = sh.from() + tid; i < sh.to(); i += THREADS) c += pair_key(Vec<T>::to(sh.row[i]), i) >= trial;
            c = warp_count(c);
            if (lane == 0) s.count[warp] = c;
            __syncthreads();
            int all = 0;
            for (int w = 0; w < WARPS; ++w) all += s.count[w];
            if (all >= top) bar = trial;
            __syncthreads();
        }
        if (tid == 0) s.n_cand = 0;
        __syncthreads();
        for (int i = sh.from() + tid; i < sh.to(); i += THREADS) {
            const uint64_t k = pair_key(Vec<T>::to(sh.row[i]), i);
            if (k >= bar) s.cand[atomicAdd(&s.n_cand, 1)] = k;         // (the keys differ: exactly `top` of them)
        }
        __syncthreads();
        n = s.n_cand;
    }
    for (int i = tid; i < top; i += THREADS)
        if (i >= n) s.best[i] = 0;
    for (int i0 = 0; i0 < n; i0 += THREADS / 2) {                      // a candidate's place: those above it, by two lanes
        const int i = i0 + tid / 2;
        const uint64_t k = i < n ? s.cand[i] : 0;
        int above = 0;
        if (i < n)
#pragma unroll 4
            for (int q = tid % 2; q < n; q += 2) above += s.cand[q] > k;
        above += __shfl_xor_sync(~0u, above, 1);
        if (i < n && tid % 2 == 0 && above < top) s.best[above] = k;
    }
    __syncthreads();
}

constexpr int RUNS = 8;                    // runs of a thread's vectors at most

struct ScoreArgs {
    Rows r;
    const int32_t *tokens;
    Window win;
    ScoreOut out;
    int32_t shift, per;                    // 2^shift blocks of a row; batches of a run
};

// One row a cluster.  2048 rows of 32 000 bf16: 28 us (4.7 TB/s; loads waited for, an exponential and seven instructions an element),
// f32 43 us (6.1 TB/s); with 64 alternatives 47 us: another eight instructions an element and five barriers a row.  Five blocks an SM
// against four: 53 and 57 us when they were compared.
template <class T, bool TOP>
__global__ void __launch_bounds__(THREADS, PER_SM) k_logprobs(const ScoreArgs a) {
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ SumSlots sl;
    const int C = 1 << a.shift, rank = blockIdx.x & (C - 1), row = blockIdx.x >> a.shift, tid = threadIdx.x;
    int token = -1;
    if (a.win.n_rows) {
        const int s = row / a.win.per_seq, j = row - s * a.win.per_seq, n = a.win.n_rows[s];
        if (j >= n) return;                                            // (all blocks of the cluster)
        if (j < n - 1) token = a.win.drafts[(size_t)s * (a.win.per_seq - 1) + j];
    } else if (a.tokens) token = a.tokens[row];
    // shared memory, with alternatives: the runs' maxima, the slots, and (rank 0) the blocks' lists
    float (*seg)[THREADS] = reinterpret_cast<float (*)[THREADS]>(dyn);
    TopSlots &ts = *reinterpret_cast<TopSlots *>(seg + RUNS);
    uint64_t *lists = reinterpret_cast<uint64_t *>(&ts + 1);
    const T *z = reinterpret_cast<const T *>(a.r.z) + (int64_t)row * a.r.ld;
    const Share<T> sh(z, a.r.vocab, rank, a.shift);
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // (peers run before their memory is written)

    const int edge = sh.edge(tid);
    const float at_edge = edge >= 0 ? Vec<T>::to(z[edge]) : 0.f, at_token = token >= 0 && token < a.r.vocab ? Vec<T>::to(z[token]) : 0.f;
    PairSums<T, true> ps;
    float most = -INFINITY;
    int left = a.per, runs = 0;
    each_vec(sh, [&](uint4 (&v)[UNROLL], int) {
        const float m = Vec<T>::max(v, UNROLL);
        ps.reach(m * LOG2E);
        ps.add(v, LOG2E);
        if (TOP) {
            most = fmaxf(most, m);
            if (--left == 0) { seg[runs++][tid] = most; most = -INFINITY; left = a.per; }
        }
    }, [&](uint4 (&v)[1], int) {
        const float m = Vec<T>::max(v, 1);
        ps.reach(m * LOG2E);
        ps.add(v, LOG2E);
        if (TOP) most = fmaxf(most, m);
    });
    const int batches = (sh.hi - sh.lo + BATCH - 1) / BATCH, all_runs = (batches + a.per - 1) / a.per;
    if (TOP && runs < all_runs) seg[runs][tid] = most;
    if (edge >= 0) ps.add(at_edge, LOG2E);
    const Sums t = row_sums<T>(ps.m, ps.S, ps.S2, sh, sl, rank, C, LOG2E, [](int) { return false; });
    const float log2S = log2f(t.S);                                    // (a row of -inf: S = 0)
    auto logp = [&](float x) { return t.S == 0.f ? -INFINITY : t.log_p(x, LOG2E, 1.f, log2S); };
    if (rank == 0 && tid == 0) {
        // (ref or m is 0)
        if (a.out.lse) a.out.lse[row] = t.S == 0.f ? -INFINITY : t.ref + fmaf(t.m, UNIT_HI, fmaf(t.m, UNIT_LO, log2S * LN2));
        const float h = log2S - t.S2 / t.S;                            // (at least 0, as log p is at most 0)
        if (a.out.entropy) a.out.entropy[row] = t.S == 0.f || h < 0.f ? 0.f : h * LN2;
        if (a.out.logp) a.out.logp[row] = token >= 0 && token < a.r.vocab ? logp(at_token) : 0.f;
    }
    if (!TOP) return;
    const int top = a.out.top;
    block_top<T>(sh, seg, all_runs, a.per * UNROLL, isnan(t.S), top, ts);
    const uint64_t *list = ts.best;
    int n = top;
    if (C > 1) {
        const uint32_t at = peer(lists + rank * top, 0);
        for (int i = tid; i < top; i += THREADS) st_peer64(at + 8 * i, ts.best[i]);
        barrier_cluster();
        if (rank) return;
        list = lists;
        n = C * top;
    }
    for (int i = tid; i < n; i += THREADS) {
        const uint64_t k = list[i];
        int above = i % top;                                           // its place in its own list
        for (int c = 0; c < C; ++c) {
            if (c == i / top) continue;
            int lo = 0, hi = top;                                      // elements of list c above it
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (list[c * top + mid] > k) lo = mid + 1; else hi = mid;
            }
            above += lo;
        }
        if (k && above < top) {
            const float v = order_value((uint32_t)(k >> 32));
            if (a.out.top_ids) a.out.top_ids[(int64_t)row * top + above] = (int32_t)~(uint32_t)k;
            if (a.out.top_logp) a.out.top_logp[(int64_t)row * top + above] = logp(v);
        }
    }
}

// ------------------------------------------------------------------ gradient of the log probabilities

struct BackArgs {
    Rows r;
    const int32_t *tokens;
    const float *lse, *entropy, *g_logp, *g_entropy, *g_lse;
    void *dz;
    int64_t ld_dz;
    int32_t shift;
};

// The vector's gradient goes where its logits were, or to a row of another alignment element by element.
template <class T>
__device__ __forceinline__ void st_grad(T *out, bool same, int j, int off, const float (&d)[Vec<T>::E]) {
    constexpr int E = Vec<T>::E;
    if (same) {
        const uint4 v = Vec<T>::pack(d);
        asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(reinterpret_cast<uint4 *>(out - off) + j), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) out[(int64_t)j * E - off + e] = Vec<T>::from(d[e]);
    }
}

// dz_v = p_v (g_lse - g_logp) - g_H p_v (log p_v + H) + [v = token] g_logp.  Elementwise: reads and writes each element once (2048
// rows of 32 000 bf16: 44 us, 5.9 TB/s).
template <class T, bool ENTROPY>
__global__ void __launch_bounds__(THREADS) k_logprobs_back(const BackArgs a) {
    constexpr int E = Vec<T>::E;
    __shared__ SumSlots sl;
    const int C = 1 << a.shift, rank = blockIdx.x & (C - 1), row = blockIdx.x >> a.shift, tid = threadIdx.x;
    const T *z = reinterpret_cast<const T *>(a.r.z) + (int64_t)row * a.r.ld;
    T *out = reinterpret_cast<T *>(a.dz) + (int64_t)row * a.ld_dz;
    const Share<T> sh(z, a.r.vocab, rank, a.shift);
    const bool same = ((uintptr_t)z & 15) == ((uintptr_t)out & 15);
    int token = a.tokens && a.g_logp ? a.tokens[row] : -1;
    if (token >= a.r.vocab) token = -1;
    const float lse = a.lse[row], gl = token >= 0 ? a.g_logp[row] : 0.f, gh = ENTROPY ? a.g_entropy[row] : 0.f;
    const float H = ENTROPY ? a.entropy[row] : 0.f, A = (a.g_lse ? a.g_lse[row] : 0.f) - gl;
    const bool none = lse == -INFINITY;                                // a row of -inf: no gradient
    float ref = lse, rest = 0.f;                                       // log p = (z - ref) - rest
    if (fabsf(lse) >= LSE_EXACT && !none) {                            // (the same in all blocks of the cluster)
        const Sums s = whole_row<T>(z, a.r.vocab, LOG2E, sl, [](int) { return false; });
        ref = s.ref; rest = log2f(s.S) * LN2;
        if (C > 1) barrier_cluster();                                  // the gradient may go where the logits are
    }
    const float c = none ? 0.f : 1.f, A1 = c * A, G1 = -c * gh, at_token = c * gl;
    auto grad = [&](float x) {
        const float l = max_nan((x - ref) - rest, FAR), p = ex2(l * LOG2E);
        return none ? 0.f : ENTROPY ? p * fmaf(G1, l + H, A1) : p * A1;
    };
    auto put = [&](const uint4 &v, int j) {
        float f[E], d[E];
        Vec<T>::unpack(v, f);
        const int i0 = j * E - sh.off;
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            f2 l = add2(add2(two(f[e], f[e + 1]), two(-ref, -ref)), two(-rest, -rest));
            float l0, l1;
            if (ENTROPY) { apart(l, l0, l1); l = two(max_nan(l0, FAR), max_nan(l1, FAR)); }
            apart(mul2(l, two(LOG2E, LOG2E)), l0, l1);
            const f2 p = two(ex2(l0), ex2(l1));
            const f2 g = ENTROPY ? fma2(two(G1, G1), add2(l, two(H, H)), two(A1, A1)) : two(A1, A1);
            apart(mul2(p, g), d[e], d[e + 1]);
        }
        if (none)
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = 0.f;
        if ((uint32_t)(token - i0) < (uint32_t)E)
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] += i0 + e == token ? at_token : 0.f;
        st_grad<T>(out, same, j, sh.off, d);
    };
    each_vec(sh, [&](uint4 (&v)[UNROLL], int j) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) put(v[u], j + u * THREADS);
    }, [&](uint4 (&v)[1], int j) { put(v[0], j); });
    if (const int i = sh.edge(tid); i >= 0) out[i] = Vec<T>::from(grad(Vec<T>::to(z[i])) + (i == token ? at_token : 0.f));
}

// ------------------------------------------------------------------ distillation

enum Mode { LOSS = 0, LOSS_GRAD = 1, GRAD = 2 };

struct DistillArgs {
    Rows r;
    Teacher t;
    float *loss, *lse, *tail_lse;
    const float *lse_in, *tail_in, *weight;
    void *dz;
    int64_t ld_dz;
    int32_t shift;
};

struct DistillSlots {
    alignas(16) int32_t id[MAX_K + 4];
    float tl[MAX_K], zk[MAX_K];            // teacher's value (-inf: no entry), from list_sums on log2 q; student's logit
    float q[MAX_K];
    uint8_t first[MAX_K];                  // 1: the first entry of its id
    unsigned long long listed[THREADS];    // a tail: which of a thread's vectors hold listed tokens
    float Q, qt, least, top, list;         // sum q, the rest, what may be rounding of it; largest listed logit, sum 2^((zk - top) scale)
    int32_t any;
};

__device__ __forceinline__ float warp_add(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
__device__ __forceinline__ float load_any(const void *p, int64_t i, int dtype) {
    return dtype == PACER_F32 ? reinterpret_cast<const float *>(p)[i]
         : dtype == PACER_BF16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(p)[i])
                               : __half2float(reinterpret_cast<const __half *>(p)[i]);
}

// The list's own sums, by one warp: q, Q, q_t, and (a tail) the listed tokens' sum of exponentials over their largest logit.
// log2 q = (t - ref) scale - log2 sum: differences of the teacher's values come first here too.  With the teacher's own log-sum-exp L at
// this temperature it is (t - L temperature) scale, the difference by one fused multiply-add.
template <bool TAIL>
__device__ __forceinline__ void list_sums(DistillSlots &ds, int K, float scale, float teacher_lse, float temp) {
    const int lane = threadIdx.x & 31;
    float top = -INFINITY, tm = -INFINITY, ref = 0.f, log2sum = 0.f;
    bool any = false;
    for (int k = lane; k < K; k += 32) {
        any |= ds.id[k] >= 0;
        if (TAIL && ds.first[k]) top = fmaxf(top, ds.zk[k]);
        if (!TAIL) tm = fmaxf(tm, ds.tl[k]);
    }
    any = __any_sync(~0u, any);
    if (TAIL) {
        if (teacher_lse == -INFINITY) log2sum = -INFINITY;             // (the teacher allows nothing)
        top = warp_max(top);
    } else {
        tm = warp_max(tm);
        ref = tm == -INFINITY ? 0.f : tm;
        float sum = 0.f;
        for (int k = lane; k < K; k += 32) sum += ex2((ds.tl[k] - ref) * scale);
        log2sum = log2f(warp_add(sum));                                // -inf: no entry that the teacher allows
    }
    const float over = top == -INFINITY ? 0.f : top;                   // (the student excludes all of them: their sum is 0)
    float Q = 0.f, list = 0.f;
    for (int k = lane; k < K; k += 32) {
        const float log2q = (TAIL ? fmaf(-teacher_lse, temp, ds.tl[k]) : ds.tl[k] - ref) * scale - log2sum;
        const float q = ds.id[k] >= 0 && log2sum != -INFINITY ? ex2(log2q) : 0.f;
        ds.tl[k] = log2q;
        ds.q[k] = q;
        Q += q;
        if (TAIL && ds.first[k]) list += ex2(max_nan((ds.zk[k] - over) * scale, FAR));
    }
    Q = warp_add(Q);
    if (TAIL) list = warp_add(list);
    if (lane == 0) {
        const float qt = TAIL ? fmaxf(0.f, 1.f - Q) : 0.f;
        // q_t where the list holds all of the teacher's mass: Q is off by 40 half steps at most (two exponentials' four, a sum's 13, and
        // three of each exponent's size, which is the list's entropy of at most ln 256 on average), the given log-sum-exp by a few of its size
        if (TAIL) ds.least = 5.9604645e-8f * fmaf(4.f, fabsf(teacher_lse), 40.f);
        ds.Q = Q + qt; ds.qt = qt; ds.top = top; ds.list = list; ds.any = any;
    }
}

// L = sum_k q_k (log q_k - log p_{id_k}) + q_t (log q_t - log p_t), p = softmax(z / temperature); q: the teacher's entries,
// renormalised (no q_t), or with the teacher's own log-sum-exp, q_t = 1 - sum q then being one class of all other tokens.
//   dL/dz_v = (p_v Q - sum_{k: id_k = v} q_k) / temperature   for the list's tokens, Q = sum q + q_t
//   dL/dz_v = w_v (Q p_t - q_t) / temperature                  for the others, w_v = p_v / p_t: their softmax among themselves
// (without q_t: p_v Q / temperature).  The tail's sum is taken over the tokens outside the list themselves (a thread knows its
// vectors with listed tokens): one minus the list's share would lose it where the student is sure of the list.
// The gradient of all others is written first, the list's tokens are put right after it.  Loss and gradient in one launch read the row
// twice, the second time out of L2: 2048 rows of 32 000 bf16 54 us (4.9 TB/s of one reading and one writing), 997 of 151 936 f32 with a
// tail 246 us (4.9 TB/s).
template <class T, bool TAIL, int MODE>
__global__ void __launch_bounds__(THREADS, PER_SM) k_distill(const DistillArgs a) {
    constexpr int E = Vec<T>::E;
    __shared__ DistillSlots ds;
    __shared__ SumSlots sl;
    const int C = 1 << a.shift, rank = blockIdx.x & (C - 1), row = blockIdx.x >> a.shift, tid = threadIdx.x, V = a.r.vocab, K = a.t.k;
    const T *z = reinterpret_cast<const T *>(a.r.z) + (int64_t)row * a.r.ld;
    const Share<T> sh(z, V, rank, a.shift);
    const float scale = LOG2E * a.t.inv_temp;
    constexpr bool marked = TAIL && MODE != GRAD;
    if (C > 1 && MODE != GRAD) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // (peers run before their memory is written)

    // the list: entry tid
    const int from = sh.from(), to = sh.to(), edge = sh.edge(tid);
    int id = -1;
    if (tid < K) {
        id = a.t.ids[(int64_t)row * K + tid];
        if (id < 0 || id >= V) id = -1;
        ds.id[tid] = id;
        ds.tl[tid] = id >= 0 ? load_any(a.t.t, (int64_t)row * K + tid, a.t.dtype) : -INFINITY;
    } else if (tid < K + 4) ds.id[tid] = -1;                           // (ids are compared four at a time)
    if (marked) ds.listed[tid] = 0;
    const float at_edge = edge >= 0 ? Vec<T>::to(z[edge]) : 0.f, my_z = id >= 0 ? Vec<T>::to(z[id]) : -INFINITY;
    __syncthreads();
    bool first = id >= 0, again = false;                               // the first entry of its id; there are more
    if (tid < K) {
#pragma unroll 4
        for (int q = 0; q < K; q += 4) {
            const int4 o = *reinterpret_cast<const int4 *>(ds.id + q);
            const bool e0 = o.x == id && q != tid, e1 = o.y == id && q + 1 != tid, e2 = o.z == id && q + 2 != tid, e3 = o.w == id && q + 3 != tid;
            again |= e0 | e1 | e2 | e3;
            first &= !((e0 && q < tid) | (e1 && q + 1 < tid) | (e2 && q + 2 < tid) | (e3 && q + 3 < tid));
        }
        ds.zk[tid] = my_z;
        ds.first[tid] = first;
    }
    const bool here = first && id >= from && id < to;
    if (marked && here) {
        const int i = (id + sh.off) / E - sh.lo;                       // its vector of the share
        if (i >= 0 && i < sh.hi - sh.lo) atomicOr(ds.listed + i % THREADS, 1ull << i / THREADS);
    }
    if (TAIL) __syncthreads();
    if (tid >= THREADS - 32) list_sums<TAIL>(ds, K, scale, TAIL ? a.t.lse[row] : 0.f, a.t.temp);     // (the warp with the fewest vectors)

    // log2 p_v = (z_v - al.ref) scale - al.m - log2 al.S; of the others among themselves (w_v) the same with ot.  m (or ref scale) and
    // log2 S are never added up: see the top of the file
    Sums al, ot;
    float al2, ot2, shift = 0.f;                                       // log2 of their sums; ot's reference over al's
    auto in_list = [&](int i) {
        bool in = false;
        if constexpr (TAIL)
            for (int k = 0; k < K; ++k) in = in || ds.id[k] == i;
        return in;
    };
    auto finish = [&]() {                                              // from the sums of the others (without a tail: of all)
        ot2 = ot.S == 0.f ? -INFINITY : log2f(ot.S);
        al = ot;
        al2 = ot2;
        if (TAIL) {                                                    // and the list's tokens
            const float d = ot.exponent(ds.top, scale);                // their largest over the others' reference
            if (d > 0.f || ot.S == 0.f) {
                al.ref = ds.top; al.m = 0.f;
                al.S = ds.list + (ot.S == 0.f ? 0.f : ex2(max_nan(ot2 - d, FAR)));
                shift = ot.S == 0.f ? 0.f : -d;
                if (ds.top == -INFINITY) al.ref = 0.f;                 // (the list's sum over 0: 0 or, of NaN, NaN)
            } else al.S = ot.S + ds.list * ex2(max_nan(d, FAR));
            al2 = al.S == 0.f ? -INFINITY : log2f(al.S);
        }
    };
    if (MODE == GRAD) {
        __syncthreads();
        const float lse = a.lse_in[row], tail = TAIL ? a.tail_in[row] : lse;
        if ((fabsf(lse) >= LSE_EXACT && lse != -INFINITY) || (fabsf(tail) >= LSE_EXACT && tail != -INFINITY)) {   // (in all blocks alike)
            ot = whole_row<T>(z, V, scale, sl, in_list);
            finish();
            if (C > 1) barrier_cluster();                              // the gradient may go where the logits are
        } else {
            // (a log-sum-exp times log2 e in two parts: its rounding would be as much again as the log-sum-exp's own)
            auto given = [&](Sums &s, float l) {
                s.m = l == -INFINITY ? 0.f : l * LOG2E;
                const float low = l == -INFINITY ? l : fmaf(l, LOG2E, -s.m);
                s.S = ex2(low);
                return low;
            };
            al2 = given(al, lse);
            ot2 = given(ot, tail);
            shift = ot.m - al.m;
        }
    } else {
        PairSums<T, false> ps;
        // A bit for each listed token of i0 .. i0 + n - 1.  K comparisons, for a vector that holds one, while its warp waits: 2048 rows of
        // 32 000 bf16, loss and gradient, 61 us with 20 ids (53 without a tail), 120 with 64 (54), 537 with 256 (82).
        auto which = [&](int i0, int n) {
            uint32_t w = 0;
            for (int q = 0; q < K; q += 4) {
                const int4 o = *reinterpret_cast<const int4 *>(ds.id + q);
                w |= (uint32_t)(o.x - i0) < (uint32_t)n ? 1u << (o.x - i0) : 0u;
                w |= (uint32_t)(o.y - i0) < (uint32_t)n ? 1u << (o.y - i0) : 0u;
                w |= (uint32_t)(o.z - i0) < (uint32_t)n ? 1u << (o.z - i0) : 0u;
                w |= (uint32_t)(o.w - i0) < (uint32_t)n ? 1u << (o.w - i0) : 0u;
            }
            return w;
        };
        unsigned long long listed = TAIL ? ds.listed[tid] : 0;
        each_vec(sh, [&](uint4 (&v)[UNROLL], int j) {
            if (TAIL) {
                if (listed & ((1u << UNROLL) - 1))
#pragma unroll
                    for (int u = 0; u < UNROLL; ++u)
                        if (listed >> u & 1) Vec<T>::hide(v[u], which((j + u * THREADS) * E - sh.off, E));
                listed >>= UNROLL;
            }
            ps.reach(Vec<T>::max(v, UNROLL) * scale);
            ps.add(v, scale);
        }, [&](uint4 (&v)[1], int j) {
            if (TAIL) {
                if (listed & 1) Vec<T>::hide(v[0], which(j * E - sh.off, E));
                listed >>= 1;
            }
            ps.reach(Vec<T>::max(v, 1) * scale);
            ps.add(v, scale);
        });
        if (edge >= 0 && (!TAIL || !which(edge, 1))) ps.add(at_edge, scale);
        ot = row_sums<T>(ps.m, ps.S, ps.S2, sh, sl, rank, C, scale, in_list);
        finish();
        if (rank == 0 && tid < 32) {
            const float it = a.t.inv_temp;
            float loss = 0.f;
            for (int k = tid; k < K; k += 32) {
                const float q = ds.q[k];
                if (q > 0.f || isnan(q)) loss += q * (ds.tl[k] * LN2 - al.log_p(ds.zk[k], scale, it, al2));
            }
            loss = warp_add(loss);
            if (tid == 0) {
                // (a student without a tail, p_t = 0 in f32: a q_t that may be rounding is none, else the loss would be infinite for it)
                const float pt2 = ot2 + shift - al2;
                if (TAIL && ds.qt > 0.f && !(pt2 < -149.f && ds.qt <= ds.least)) loss += ds.qt * (log2f(ds.qt) - pt2) * LN2;
                if (a.loss) a.loss[row] = ds.any && al2 != -INFINITY ? loss : 0.f;
                // ref or m is 0; ref goes by the same 1 / temperature as the exponents.  (LOWEST where a finite log-sum-exp is out of
                // range: -inf says that nothing is left)
                const float it_hi = scale * UNIT_HI, it_lo = fmaf(scale, UNIT_HI, -it_hi) + scale * UNIT_LO;
                auto whole = [&](const Sums &s, float log2S) {
                    const float l = fmaf(s.ref, it_hi, fmaf(s.ref, it_lo, fmaf(s.m, UNIT_HI, fmaf(s.m, UNIT_LO, log2S * LN2))));
                    return log2S == -INFINITY ? log2S : max_nan(l, LOWEST);
                };
                if (a.lse) a.lse[row] = whole(al, al2);
                if (TAIL && a.tail_lse) a.tail_lse[row] = whole(ot, ot2);
            }
        }
    }
    if (MODE == LOSS) return;

    T *out = reinterpret_cast<T *>(a.dz) + (int64_t)row * a.ld_dz;
    const bool same = ((uintptr_t)z & 15) == ((uintptr_t)out & 15), none = !ds.any || al2 == -INFINITY, others = !none && (ot2 != -INFINITY || isnan(al2));
    const float g = a.weight[row] * a.t.inv_temp;
    // (w_v = 2^t / S; two roundings of the quotient at most: S is at least about 1 and below 2^35)
    const float coef = __fdividef(!TAIL ? g * ds.Q : g * (ds.Q * ex2(max_nan(ot2 + shift - al2, FAR)) - ds.qt), ot.S);
    const f2 c0 = two(-ot.ref, -ot.ref), c1 = two(scale, scale), c2 = two(-ot.m, -ot.m), c3 = two(coef, coef);
    auto put = [&](const uint4 &v, int j) {
        float f[E], d[E];
        Vec<T>::unpack(v, f);
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            float t0, t1;
            apart(fma2(add2(two(f[e], f[e + 1]), c0), c1, c2), t0, t1);
            apart(mul2(two(ex2(t0), ex2(t1)), c3), d[e], d[e + 1]);
        }
        if (!others)
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] = 0.f;
        st_grad<T>(out, same, j, sh.off, d);
    };
    each_vec_back(sh, [&](uint4 (&v)[UNROLL], int j) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) put(v[u], j + u * THREADS);
    }, [&](uint4 (&v)[1], int j) { put(v[0], j); });
    if (edge >= 0) out[edge] = Vec<T>::from(others ? coef * ex2(ot.exponent(at_edge, scale)) : 0.f);
    __syncthreads();
    if (here) {                                                        // the list's tokens
        float qs = ds.q[tid];
        if (again)
            for (int k = tid + 1; k < K; ++k) qs += ds.id[k] == id ? ds.q[k] : 0.f;
        out[id] = Vec<T>::from(none ? 0.f : g * (ds.Q * ex2(max_nan(al.exponent(my_z, scale) - al2, FAR)) - qs));
    }
}

// ------------------------------------------------------------------ launches

static int elem_bytes(int dtype) { return dtype == PACER_F32 ? 4 : 2; }

// Blocks per row (log2).  More than one while two blocks an SM take all rows' and a thread keeps a vector, or all block slots do and a
// block keeps 64 KB: one row of 151 936 f32 with 20 alternatives takes 12.2 us by eight blocks, 13.5 by four, 24.6 by one; 200 such rows
// 32.5 us by two, 45.5 by one; 136 rows of 32 256 bf16 10.0 by two, 11.7 by four; 300 rows of 32 000 bf16 11.8 by one, 13.7 by two.
// And, where rows are read twice, while the rows at work (of all SMs) exceed what L2 (126 MB) surely keeps: 997 rows of 151 936 f32,
// loss and gradient, took 257 us with eight blocks a row (56 MB at work), 288 us with four (112 MB).
static int blocks_per_row_log2(int rows, int vocab, int elem, bool twice) {
    const int slots = PER_SM * 148;
    const double bytes = (double)vocab * elem;
    int shift = 0;
    for (; 1 << shift < MAX_C; ++shift) {
        const int64_t blocks = (int64_t)rows << (shift + 1);
        const double share = bytes / (2 << shift);
        if (!((blocks <= 2 * 148 && share >= THREADS * 16) || (blocks <= slots && share >= 65536) ||
              (twice && std::min(rows, slots >> shift) * bytes > 64e6))) break;
    }
    return shift;
}

template <auto K, class A>
static cudaError_t launch(const A &a, size_t smem, cudaStream_t st) {
    const int C = 1 << a.shift;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)a.r.rows * (unsigned)C);
    c.blockDim = dim3(THREADS);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = C; at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    c.attrs = at;
    c.numAttrs = C > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&c, K, a);
}

// f(a value of the rows' element type)
template <class F>
static cudaError_t by_type(int dtype, F f) {
    return dtype == PACER_F32 ? f(float()) : dtype == PACER_BF16 ? f(__nv_bfloat16()) : f(__half());
}

cudaError_t logprobs(const Rows &r, const int32_t *tokens, const Window &win, const ScoreOut &out, cudaStream_t st) {
    const int elem = elem_bytes(r.dtype), shift = blocks_per_row_log2(r.rows, r.vocab, elem, false);
    const int batches = ((r.vocab * elem / 16 + 2 >> shift) + BATCH) / BATCH;
    const ScoreArgs a{r, tokens, win, out, shift, std::max(1, (batches + RUNS - 1) / RUNS)};
    const size_t smem = out.top == 0 ? 0 : RUNS * THREADS * 4 + sizeof(TopSlots) + ((size_t)out.top * 8 << shift);
    return by_type(r.dtype, [&](auto t) {
        using T = decltype(t);
        return out.top > 0 ? launch<k_logprobs<T, true>>(a, smem, st) : launch<k_logprobs<T, false>>(a, smem, st);
    });
}

cudaError_t logprobs_backward(const Rows &r, const int32_t *tokens, const float *lse, const float *entropy, const float *g_logp,
                              const float *g_entropy, const float *g_lse, void *dz, int64_t ld_dz, cudaStream_t st) {
    const BackArgs a{r, tokens, lse, entropy, g_logp, g_entropy, g_lse, dz, ld_dz, blocks_per_row_log2(r.rows, r.vocab, elem_bytes(r.dtype), false)};
    return by_type(r.dtype, [&](auto t) {
        using T = decltype(t);
        return g_entropy ? launch<k_logprobs_back<T, true>>(a, 0, st) : launch<k_logprobs_back<T, false>>(a, 0, st);
    });
}

template <int MODE>
static cudaError_t distill_mode(DistillArgs &a, cudaStream_t st) {
    const int elem = elem_bytes(a.r.dtype);
    a.shift = blocks_per_row_log2(a.r.rows, a.r.vocab, elem, MODE == LOSS_GRAD);
    // (a tail: a thread has a bit for each of its vectors, 64 at most; MAX_VOCAB f32 over MAX_C blocks are 48)
    while (a.t.lse && (a.r.vocab * elem / 16 + 2 >> a.shift) + 1 > 64 * THREADS) ++a.shift;
    return by_type(a.r.dtype, [&](auto t) {
        using T = decltype(t);
        return a.t.lse ? launch<k_distill<T, true, MODE>>(a, 0, st) : launch<k_distill<T, false, MODE>>(a, 0, st);
    });
}

cudaError_t distill(const Rows &r, const Teacher &t, float *loss, float *lse, float *tail_lse, const float *weight, void *dz, int64_t ld_dz,
                    cudaStream_t st) {
    DistillArgs a{r, t, loss, lse, tail_lse, nullptr, nullptr, weight, dz, ld_dz, 0};
    return dz ? distill_mode<LOSS_GRAD>(a, st) : distill_mode<LOSS>(a, st);
}

cudaError_t distill_backward(const Rows &r, const Teacher &t, const float *lse, const float *tail_lse, const float *weight, void *dz,
                             int64_t ld_dz, cudaStream_t st) {
    DistillArgs a{r, t, nullptr, nullptr, nullptr, lse, tail_lse, weight, dz, ld_dz, 0};
    return distill_mode<GRAD>(a, st);
}

}  // namespace lg

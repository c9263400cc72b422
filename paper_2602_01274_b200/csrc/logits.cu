// Operators on rows of logits: log probabilities of given tokens with entropy and the best alternatives, distillation from a
// teacher's top logits, and their gradients.
//
// All are bound by HBM: a row is read once (and its gradient written once).  A row belongs to a cluster of C blocks, each with a
// share of its 16-byte vectors, so that one row can have the loads of up to 16 SMs in flight; with many rows C is 1.
// Softmax sums are held as (m, S) with S = sum 2^((z - m) scale): the reference m is raised only when a logit lies more than
// 2^SLACK above it (S stays below vocab * 2^SLACK), so that the common path has no rescaling.  z - m is taken first: logits of any
// size (a row masked with the type's lowest value among them) keep their differences.
#include "logits.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/pacer.h"

namespace lg {

constexpr int THREADS = 256, WARPS = THREADS / 32, MAX_C = 8;
constexpr int UNROLL = 4;                  // 16-byte loads in flight per thread
constexpr int CAND = 1280;                 // candidates for the alternatives that a block collects at most
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float NO_REF = -3.402823466e38f, SLACK = 16.f;
constexpr float FAR = -1000.f;             // exponents are cut here: 2^FAR is 0, and 0 * FAR too
constexpr float LSE_EXACT = 65536.f;       // beyond it an f32 log-sum-exp no longer tells the logits of a row apart

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

    __device__ Share(const T *row_, int vocab_, int rank, int C) : row(row_), vocab(vocab_) {
        off = (int)(((uintptr_t)row & 15) / sizeof(T));
        const int nv = (int)(((int64_t)off + vocab + E - 1) / E);
        lo = (int)((int64_t)nv * rank / C);
        hi = (int)((int64_t)nv * (rank + 1) / C);
        first = last = -1;
        if (lo < hi && lo == 0 && (off || vocab < E)) first = lo++;
        if (lo < hi && hi == nv && ((int64_t)off + vocab) % E) last = --hi;
    }
    __device__ const uint4 *vecs() const { return reinterpret_cast<const uint4 *>(row - off); }
    __device__ int begin(int j) const { return max(j * E - off, 0); }
    __device__ int end(int j) const { return (int)min((int64_t)(j + 1) * E - off, (int64_t)vocab); }
    // elements of the block: [from, to)
    __device__ int from() const { return first >= 0 ? begin(first) : begin(lo); }
    __device__ int to() const { return last >= 0 ? end(last) : hi > lo ? end(hi - 1) : first >= 0 ? end(first) : from(); }
};

__device__ __forceinline__ uint4 ld_row(const uint4 *p) {        // (not the read-only path: a gradient may go where its logits were)
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
// A thread's UNROLL vectors of a batch: j, j + THREADS, ..; past the block's share -inf.
template <class T>
__device__ __forceinline__ void ld_batch(const Share<T> &sh, int j, uint4 (&v)[UNROLL]) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
        v[u] = j + u * THREADS < sh.hi ? ld_row(sh.vecs() + j + u * THREADS) : make_uint4(Vec<T>::NONE, Vec<T>::NONE, Vec<T>::NONE, Vec<T>::NONE);
}
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

// S = sum 2^t, S2 = sum 2^t t with t = (z - m) scale.  A logit of -inf adds nothing; NaN and +inf make the sums NaN.
struct Sums {
    float m = NO_REF, S = 0.f, S2 = 0.f;
    __device__ void raise(float to, float scale) {
        const float d = fmaxf((m - to) * scale, FAR), r = ex2(d);
        S2 = r * fmaf(S, d, S2);
        S *= r;
        m = to;
    }
    __device__ void add(float z, float scale) {
        if (z > m) raise(z, scale);
        const float t = max_nan((z - m) * scale, FAR), x = ex2(t);
        S += x;
        S2 = fmaf(x, t, S2);
    }
    __device__ void join(float m2, float s, float s2, float scale) {   // with the sums of another share
        const float to = fmaxf(m, m2);
        raise(to, scale);
        const float d = fmaxf((m2 - to) * scale, FAR), r = ex2(d);
        S = fmaf(r, s, S);
        S2 = fmaf(r, fmaf(s, d, s2), S2);
    }
};

// A thread's sums while it reads its vectors: even and odd elements apart.
template <bool ENTROPY>
struct PairSums {
    float m = NO_REF;
    f2 S = 0, S2 = 0;
    // `top`: the largest of the elements that come next
    __device__ void reach(float top, float scale, float slack) {
        if (top > m + slack) {
            const float d = fmaxf((m - top) * scale, FAR), r = ex2(d);
            if (ENTROPY) S2 = mul2(two(r, r), fma2(S, two(d, d), S2));
            S = mul2(two(r, r), S);
            m = top;
        }
    }
    template <int E>
    __device__ void add(const float (&f)[E], float scale) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            f2 t = mul2(add2(two(f[e], f[e + 1]), two(-m, -m)), two(scale, scale));
            float t0, t1;
            apart(t, t0, t1);
            if (ENTROPY) { t0 = max_nan(t0, FAR); t1 = max_nan(t1, FAR); t = two(t0, t1); }      // (0 * -inf; without the product 2^-inf does)
            const f2 x = two(ex2(t0), ex2(t1));
            S = add2(S, x);
            if (ENTROPY) S2 = fma2(x, t, S2);
        }
    }
    __device__ Sums sums() const {
        Sums s;
        float a, b;
        s.m = m;
        apart(S, a, b); s.S = a + b;
        if (ENTROPY) { apart(S2, a, b); s.S2 = a + b; }
        return s;
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

struct SumSlots {
    float warp[WARPS][3], block[MAX_C][3];
};
// The row's sums in every thread of every block of the cluster; fixed order.  Ends with the cluster (or block) in step.
__device__ __forceinline__ Sums row_sums(Sums s, SumSlots &sl, int rank, int C, float scale) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float m = __shfl_xor_sync(~0u, s.m, o), a = __shfl_xor_sync(~0u, s.S, o), b = __shfl_xor_sync(~0u, s.S2, o);
        s.join(m, a, b, scale);
    }
    if (lane == 0) { sl.warp[warp][0] = s.m; sl.warp[warp][1] = s.S; sl.warp[warp][2] = s.S2; }
    __syncthreads();
    Sums t;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) t.join(sl.warp[w][0], sl.warp[w][1], sl.warp[w][2], scale);
    if (C == 1) return t;
    if ((int)threadIdx.x < C) {
        const uint32_t at = peer(&sl.block[rank][0], threadIdx.x);
        st_peer(at, t.m); st_peer(at + 4, t.S); st_peer(at + 8, t.S2);
    }
    barrier_cluster();
    Sums u;
    for (int c = 0; c < C; ++c) u.join(sl.block[c][0], sl.block[c][1], sl.block[c][2], scale);
    return u;
}

// The sums of a whole row in every thread of one block, element by element, without the tokens that skip() names: for rows whose
// log-sum-exp says too little (see LSE_EXACT).
template <class T, class Skip>
__device__ Sums whole_row(const T *z, int vocab, float scale, SumSlots &sl, Skip skip) {
    Sums s;
    for (int i = threadIdx.x; i < vocab; i += THREADS)
        if (!skip(i)) s.add(Vec<T>::to(z[i]), scale);
    __syncwarp();
    return row_sums(s, sl, 0, 1, scale);
}

// ------------------------------------------------------------------ alternatives

// Order of the alternatives: larger logit first, then the lower index; NaN last.  A logit as an integer of that order (0: NaN):
__device__ __forceinline__ uint32_t order_key(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);                       // -0 and 0 are equal
    return isnan(z) ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float order_value(uint32_t k) { return __uint_as_float(k == 0u ? 0x7fffffffu : (k & 0x80000000u) ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ uint64_t pair_key(float z, int idx) { return ((uint64_t)order_key(z) << 32) | (uint32_t)~idx; }

constexpr int SEGS = 16, FLAGS = 1024;     // a thread's vectors in at most SEGS runs of whole batches; runs that are read again

struct TopSlots {
    float seg[SEGS][THREADS];              // largest value of each run
    uint32_t key[THREADS];
    int32_t vec[THREADS];
    uint64_t cand[CAND], best[MAX_TOP];
    uint16_t flagged[FLAGS];
    int32_t n_flag, n_cand, bound_idx, ties;
    uint32_t bound;
    int32_t count[WARPS];
};

__device__ __forceinline__ int warp_count(int v) { return __reduce_add_sync(~0u, v); }

// The `top` best elements of the block's share, in order, to best[] (with fewer elements: all, the rest 0).  Thread tid has read the
// whole vectors lo + tid, lo + tid + THREADS, .. in `segs` runs of `run` vectors, whose largest values are in seg[][tid].
// The top-th best of the 256 per-thread maxima bounds the top-th best element from below; only the runs that reach the bound are
// read again, out of L2 (2048 rows of 32 003 bf16, top 64: about 70 runs of four vectors of 4000, 74 candidates).
template <class T>
__device__ void block_top(const Share<T> &sh, int segs, int run, bool has_nan, int top, TopSlots &s) {
    constexpr int E = Vec<T>::E, N = THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool mine = sh.lo + tid < sh.hi;
    float bv = -INFINITY;
    int bseg = 0;
    for (int g = 0; g < segs; ++g) {
        const float v = s.seg[g][tid];
        if (v > bv) { bv = v; bseg = g; }
    }
    // (a maximum that ignores NaN says nothing certain about a thread that saw only -inf: it then counts as lowest)
    const uint32_t key = !mine || (has_nan && bv == -INFINITY) ? 0u : order_key(bv);
    s.key[tid] = key;
    if (tid == 0) { s.n_flag = s.n_cand = s.ties = 0; s.bound = 0; s.bound_idx = INT32_MAX; }
    __syncthreads();
    if (warp == 0 && min(sh.hi - sh.lo, THREADS) >= top) {
        uint32_t k[N], hi = 0, lo = ~0u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            k[i] = s.key[i * 32 + lane];
            if (i * 32 + lane < sh.hi - sh.lo) { hi = max(hi, k[i]); lo = min(lo, k[i]); }
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
        int at = INT32_MAX;
        if (key == bound) {
            const int j0 = sh.lo + tid + bseg * run * THREADS;
            for (int i = 0; i < run && at == INT32_MAX && j0 + i * THREADS < sh.hi; ++i) {
                const uint4 v = ld_row(sh.vecs() + j0 + i * THREADS);
                if (Vec<T>::max(&v, 1) == bv) at = j0 + i * THREADS;
            }
        }
        s.vec[tid] = at;
        __syncthreads();
        if (warp == 0) {
            int v[N], lim = 0;                                         // least vector number with `ties` of them at most there
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = s.vec[i * 32 + lane];
            for (int b = 31 - __clz(sh.hi); b >= 0; --b) {
                const int trial = lim | (1 << b);
                int n = 0;
#pragma unroll
                for (int i = 0; i < N; ++i) n += v[i] < trial;
                if (warp_count(n) < s.ties) lim = trial;
            }
            if (lane == 0) s.bound_idx = sh.end(min(lim, sh.hi - 1)) - 1;
        }
        __syncthreads();
    }
    const int bound_idx = s.bound_idx;
    const uint64_t least = ((uint64_t)bound << 32) | (uint32_t)~bound_idx;
    if (mine)
        for (int g = 0; g < segs; ++g) {
            const float v = s.seg[g][tid];
            const int j = sh.lo + tid + g * run * THREADS;
            if (j < sh.hi && ((has_nan && v == -INFINITY) || order_key(v) > bound || (order_key(v) == bound && sh.begin(j) <= bound_idx))) {
                const int at = atomicAdd(&s.n_flag, 1);
                if (at < FLAGS) s.flagged[at] = (uint16_t)(g * THREADS + tid);
            }
        }
    __syncthreads();
    const int nf = s.n_flag;
    auto test = [&](float z, int i) {
        const uint64_t k = pair_key(z, i);
        if (k >= least) {
            const int at = atomicAdd(&s.n_cand, 1);
            if (at < CAND) s.cand[at] = k;
        }
    };
    if (nf <= FLAGS) {
        for (int w = tid; w < nf * run; w += THREADS) {
            const int f = s.flagged[w / run], j = sh.lo + f % THREADS + ((f / THREADS) * run + w % run) * THREADS;
            if (j < sh.hi) {
                const uint4 v = ld_row(sh.vecs() + j);
                if (has_nan || order_key(Vec<T>::max(&v, 1)) >= bound) {
                    float x[E];
                    Vec<T>::unpack(v, x);
#pragma unroll
                    for (int e = 0; e < E; ++e) test(x[e], sh.begin(j) + e);
                }
            }
        }
        if (tid < 2) {
            const int j = tid ? sh.last : sh.first;
            if (j >= 0)
                for (int i = sh.begin(j); i < sh.end(j); ++i) test(Vec<T>::to(sh.row[i]), i);
        }
    }
    __syncthreads();
    int n = s.n_cand;
    if (n > CAND || nf > FLAGS) {                                      // (many elements of few threads, or NaN): bit by bit
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
    for (int i0 = 0; i0 < n; i0 += THREADS / 4) {                      // a candidate's place: those above it, by four lanes
        const int i = i0 + tid / 4;
        const uint64_t k = i < n ? s.cand[i] : 0;
        int above = 0;
        if (i < n)
            for (int q = tid % 4; q < n; q += 4) above += s.cand[q] > k;
        above += __shfl_xor_sync(~0u, above, 1);
        above += __shfl_xor_sync(~0u, above, 2);
        if (i < n && tid % 4 == 0 && above < top) s.best[above] = k;
    }
    __syncthreads();
}

struct ScoreArgs {
    Rows r;
    const int32_t *tokens;
    Window win;
    ScoreOut out;
    int32_t C;
};

template <class T, bool TOP>
__global__ void __launch_bounds__(THREADS, 4) k_logprobs(const ScoreArgs a) {
    constexpr int E = Vec<T>::E;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ SumSlots sl;
    const int C = a.C, rank = blockIdx.x % C, row = blockIdx.x / C, tid = threadIdx.x;
    int token = -1;
    if (a.win.n_rows) {
        const int s = row / a.win.per_seq, j = row - s * a.win.per_seq, n = a.win.n_rows[s];
        if (j >= n) return;                                            // (all blocks of the cluster)
        if (j < n - 1) token = a.win.drafts[(size_t)s * (a.win.per_seq - 1) + j];
    } else if (a.tokens) token = a.tokens[row];
    const T *z = reinterpret_cast<const T *>(a.r.z) + (int64_t)row * a.r.ld;
    const Share<T> sh(z, a.r.vocab, rank, C);
    if (C > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // (peers run before their memory is written)

    TopSlots &ts = *reinterpret_cast<TopSlots *>(dyn);
    const int batches = (sh.hi - sh.lo + UNROLL * THREADS - 1) / (UNROLL * THREADS), per = (batches + SEGS - 1) / SEGS;      // a run: `per` batches
    PairSums<true> ps;
    float most = -INFINITY;
    for (int n = 0, left = per, g = 0; n < batches; ++n) {
        uint4 v[UNROLL];
        ld_batch(sh, sh.lo + tid + n * UNROLL * THREADS, v);
        const float m = Vec<T>::max(v, UNROLL);
        ps.reach(m, LOG2E, SLACK * LN2);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            float f[E];
            Vec<T>::unpack(v[u], f);
            ps.add(f, LOG2E);
        }
        if (TOP) {
            most = fmaxf(most, m);
            if (--left == 0 || n == batches - 1) { ts.seg[g++][tid] = most; most = -INFINITY; left = per; }
        }
    }
    Sums s = ps.sums();
    if (tid < 2) {
        const int p = tid ? sh.last : sh.first;
        if (p >= 0)
            for (int i = sh.begin(p); i < sh.end(p); ++i) s.add(Vec<T>::to(z[i]), LOG2E);
    }
    __syncwarp();
    if (C > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    const Sums t = row_sums(s, sl, rank, C, LOG2E);
    const float log2S = log2f(t.S), logS = log2S * LN2;                // (a row of -inf: S = 0)
    auto logp = [&](float x) { return t.S == 0.f ? -INFINITY : (x - t.m) - logS; };
    if (rank == 0 && tid == 0) {
        if (a.out.lse) a.out.lse[row] = t.S == 0.f ? -INFINITY : t.m + logS;
        if (a.out.entropy) a.out.entropy[row] = t.S == 0.f ? 0.f : (log2S - t.S2 / t.S) * LN2;
        if (a.out.logp) a.out.logp[row] = token >= 0 && token < a.r.vocab ? logp(Vec<T>::to(z[token])) : 0.f;
    }
    if (!TOP) return;
    uint64_t *lists = reinterpret_cast<uint64_t *>(dyn + sizeof(TopSlots));            // rank 0: the blocks' lists
    const int top = a.out.top;
    block_top<T>(sh, per ? (batches + per - 1) / per : 0, per * UNROLL, isnan(t.S), top, ts);
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
    int32_t C;
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

// dz_v = p_v (g_lse - g_logp) - g_H p_v (log p_v + H) + [v = token] g_logp.  Elementwise: reads and writes each element once.
template <class T, bool ENTROPY>
__global__ void __launch_bounds__(THREADS) k_logprobs_back(const BackArgs a) {
    constexpr int E = Vec<T>::E;
    __shared__ SumSlots sl;
    const int C = a.C, rank = blockIdx.x % C, row = blockIdx.x / C, tid = threadIdx.x;
    const T *z = reinterpret_cast<const T *>(a.r.z) + (int64_t)row * a.r.ld;
    T *out = reinterpret_cast<T *>(a.dz) + (int64_t)row * a.ld_dz;
    const Share<T> sh(z, a.r.vocab, rank, C);
    const bool same = ((uintptr_t)z & 15) == ((uintptr_t)out & 15);
    int token = a.tokens && a.g_logp ? a.tokens[row] : -1;
    if (token >= a.r.vocab) token = -1;
    const float lse = a.lse[row], gl = token >= 0 ? a.g_logp[row] : 0.f, gh = ENTROPY ? a.g_entropy[row] : 0.f;
    const float H = ENTROPY ? a.entropy[row] : 0.f, A = (a.g_lse ? a.g_lse[row] : 0.f) - gl;
    const bool none = lse == -INFINITY;                                // a row of -inf: no gradient
    float ref = lse, rest = 0.f;                                       // log p = (z - ref) - rest
    if (fabsf(lse) >= LSE_EXACT && !none) {                            // (the same in all blocks of the cluster)
        const Sums s = whole_row(z, a.r.vocab, LOG2E, sl, [](int) { return false; });
        ref = s.m; rest = log2f(s.S) * LN2;
        if (C > 1) barrier_cluster();                                  // the gradient may go where the logits are
    }
    const float c = none ? 0.f : 1.f, A1 = c * A, G1 = -c * gh, at_token = c * gl;
    auto grad = [&](float x) {
        const float l = max_nan((x - ref) - rest, FAR), p = ex2(l * LOG2E);
        return none ? 0.f : ENTROPY ? p * fmaf(G1, l + H, A1) : p * A1;
    };
    for (int j = sh.lo + tid; j < sh.hi; j += UNROLL * THREADS) {
        uint4 v[UNROLL];
        ld_batch(sh, j, v);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (j + u * THREADS >= sh.hi) break;
            float f[E], d[E];
            Vec<T>::unpack(v[u], f);
            const int i0 = (j + u * THREADS) * E - sh.off;
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
            st_grad<T>(out, same, j + u * THREADS, sh.off, d);
        }
    }
    if (tid < 2) {
        const int p = tid ? sh.last : sh.first;
        if (p >= 0)
            for (int i = sh.begin(p); i < sh.end(p); ++i) out[i] = Vec<T>::from(grad(Vec<T>::to(z[i])) + (i == token ? at_token : 0.f));
    }
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
    int32_t C;
};

struct DistillSlots {
    SumSlots sums;
    int32_t id[MAX_K];
    float q[MAX_K];
    float red[WARPS];
};

__device__ __forceinline__ float block_add(float v, float *red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    __syncthreads();
    if (lane == 0) red[warp] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) t += red[w];
    return t;
}
__device__ __forceinline__ float block_max(float v, float *red) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    __syncthreads();
    if (lane == 0) red[warp] = v;
    __syncthreads();
    float t = red[0];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) t = fmaxf(t, red[w]);
    return t;
}
__device__ __forceinline__ float load_any(const void *p, int64_t i, int dtype) {
    return dtype == PACER_F32 ? reinterpret_cast<const float *>(p)[i]
         : dtype == PACER_BF16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(p)[i])
                               : __half2float(reinterpret_cast<const __half *>(p)[i]);
}

// L = sum_k q_k (log q_k - log p_{id_k}) + q_t (log q_t - log p_t), p = softmax(z / temperature); q: the teacher's entries,
// renormalised (no q_t), or with the teacher's own log-sum-exp, q_t = 1 - sum q then being one class of all other tokens.
//   dL/dz_v = (p_v Q - sum_{k: id_k = v} q_k) / temperature   for the list's tokens, Q = sum q + q_t
//   dL/dz_v = w_v (Q p_t - q_t) / temperature                  for the others, w_v = p_v / p_t: their softmax among themselves
// (without q_t: p_v Q / temperature).  The tail's sum is taken over the tokens outside the list themselves, marked in a bitmap:
// one minus the list's share would lose it where the student is sure of the list.
// The gradient is written from a second reading of the row, out of L2, with the list's tokens put right after it.
template <class T, bool TAIL, int MODE>
__global__ void __launch_bounds__(THREADS, 4) k_distill(const DistillArgs a) {
    constexpr int E = Vec<T>::E;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ DistillSlots ds;
    const int C = a.C, rank = blockIdx.x % C, row = blockIdx.x / C, tid = threadIdx.x, V = a.r.vocab, K = a.t.k;
    const T *z = reinterpret_cast<const T *>(a.r.z) + (int64_t)row * a.r.ld;
    const Share<T> sh(z, V, rank, C);
    const float scale = LOG2E * a.t.inv_temp;
    if (C > 1 && MODE != GRAD) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");

    // the list: entry tid
    uint32_t *marks = reinterpret_cast<uint32_t *>(dyn);               // TAIL: a bit per element of the block's share
    const int from = sh.from(), to = sh.to();
    if (TAIL && MODE != GRAD)
        for (int i = tid; i < (to - from + 31) / 32 + 1; i += THREADS) marks[i] = 0;
    int id = -1;
    float tl = -INFINITY, zk = -INFINITY;
    if (tid < K) {
        id = a.t.ids[(int64_t)row * K + tid];
        if (id < 0 || id >= V) id = -1;
        if (id >= 0) {
            tl = load_any(a.t.t, (int64_t)row * K + tid, a.t.dtype) * scale;
            zk = Vec<T>::to(z[id]);
        }
        ds.id[tid] = id;
    }
    float norm;                                                        // log2 of the teacher's sum
    if (TAIL) norm = a.t.lse[row] * LOG2E;
    else {
        const float m = block_max(tl, ds.red), ref = m == -INFINITY ? 0.f : m;
        norm = ref + log2f(block_add(ex2(tl - ref), ds.red));          // -inf: an empty list
    }
    const float lq = id >= 0 ? tl - norm : -INFINITY, q = id >= 0 && norm != -INFINITY ? ex2(lq) : 0.f;
    bool first = id >= 0;
    __syncthreads();
    if (id >= 0) {
        for (int k = 0; k < tid; ++k) first = first && ds.id[k] != id;
        ds.q[tid] = q;
        if (TAIL && MODE != GRAD && id >= from && id < to) atomicOr(marks + ((id - from) >> 5), 1u << ((id - from) & 31));
    } else if (tid < K) ds.q[tid] = 0.f;
    float Q = block_add(q, ds.red);                                    // (and the marks are set)
    const float qt = TAIL ? fmaxf(0.f, 1.f - Q) : 0.f;
    const bool any = __syncthreads_or(id >= 0);
    Q += qt;

    // log p_v = (z_v - ref) inv_temp - all, of the others among themselves: (z_v - tref) inv_temp - tail
    float ref, all, tref, tail;
    const float it = a.t.inv_temp, slack = SLACK / scale;
    auto in_list = [&](int i) {
        for (int k = 0; k < K; ++k)
            if (ds.id[k] == i) return true;
        return false;
    };
    auto finish = [&](const Sums &t) {                                 // from the sums of the others (without a tail: of all)
        ref = tref = t.m;
        tail = t.S == 0.f ? -INFINITY : log2f(t.S) * LN2;
        all = tail;
        if (TAIL) {                                                    // and the list's tokens
            const float top = block_max(first ? zk : -INFINITY, ds.red);
            if (top > ref) ref = top;
            const float others = t.S == 0.f ? 0.f : ex2(max_nan(((tref - ref) * it + tail) * LOG2E, FAR));
            all = log2f(block_add(first ? ex2(max_nan((zk - ref) * scale, FAR)) : 0.f, ds.red) + others) * LN2;
        }
    };
    if (MODE == GRAD) {
        ref = tref = 0.f;
        all = a.lse_in[row];
        tail = TAIL ? a.tail_in[row] : all;
        if ((fabsf(all) >= LSE_EXACT && all != -INFINITY) || (fabsf(tail) >= LSE_EXACT && tail != -INFINITY)) {   // (in all blocks alike)
            finish(whole_row(z, V, scale, ds.sums, [&](int i) { return TAIL && in_list(i); }));
            if (C > 1) barrier_cluster();                              // the gradient may go where the logits are
        }
    } else {
        PairSums<false> ps;
        for (int j = sh.lo + tid; j < sh.hi; j += UNROLL * THREADS) {
            uint4 v[UNROLL];
            ld_batch(sh, j, v);
            if (TAIL)
#pragma unroll
                for (int u = 0; u < UNROLL; ++u) {
                    if (j + u * THREADS >= sh.hi) break;
                    const int o = (j + u * THREADS) * E - sh.off - from;
                    const uint32_t w = __funnelshift_r(marks[o >> 5], marks[(o >> 5) + 1], o & 31) & ((1u << E) - 1);
                    if (w) Vec<T>::hide(v[u], w);
                }
            ps.reach(Vec<T>::max(v, UNROLL), scale, slack);
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                float f[E];
                Vec<T>::unpack(v[u], f);
                ps.add(f, scale);
            }
        }
        Sums s = ps.sums();
        if (tid < 2) {
            const int p = tid ? sh.last : sh.first;
            if (p >= 0)
                for (int i = sh.begin(p); i < sh.end(p); ++i)
                    if (!TAIL || !(marks[(i - from) >> 5] >> ((i - from) & 31) & 1)) s.add(Vec<T>::to(z[i]), scale);
        }
        __syncwarp();
        if (C > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        finish(row_sums(s, ds.sums, rank, C, scale));
        float loss = block_add(q > 0.f ? q * (lq * LN2 - ((zk - ref) * it - all)) : 0.f, ds.red);
        if (rank == 0 && tid == 0) {
            if (TAIL && qt > 0.f) loss += qt * (log2f(qt) * LN2 - ((tref - ref) * it + tail - all));
            if (a.loss) a.loss[row] = any && all != -INFINITY ? loss : 0.f;
            // (NO_REF where a finite one is out of range: -inf says that nothing is left)
            if (a.lse) a.lse[row] = all == -INFINITY ? all : max_nan(ref * it + all, NO_REF);
            if (TAIL && a.tail_lse) a.tail_lse[row] = tail == -INFINITY ? tail : max_nan(tref * it + tail, NO_REF);
        }
    }
    if (MODE == LOSS) return;

    T *out = reinterpret_cast<T *>(a.dz) + (int64_t)row * a.ld_dz;
    const bool same = ((uintptr_t)z & 15) == ((uintptr_t)out & 15), none = !any || all == -INFINITY;
    const float g = a.weight[row] * it;
    const bool others = !none && tail != -INFINITY;
    const float coef = !others ? 0.f : g * (TAIL ? Q * ex2(max_nan(((tref - ref) * it + tail - all) * LOG2E, FAR)) - qt : Q), off = others ? tail : 0.f;
    auto grad = [&](float x) { return others ? coef * ex2(((x - tref) * it - off) * LOG2E) : 0.f; };
    const float c1 = it * LOG2E, c2 = -off * LOG2E;
    for (int j = sh.lo + tid; j < sh.hi; j += UNROLL * THREADS) {
        uint4 v[UNROLL];
        ld_batch(sh, j, v);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (j + u * THREADS >= sh.hi) break;
            float f[E], d[E];
            Vec<T>::unpack(v[u], f);
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                float t0, t1;
                apart(fma2(add2(two(f[e], f[e + 1]), two(-tref, -tref)), two(c1, c1), two(c2, c2)), t0, t1);
                apart(mul2(two(ex2(t0), ex2(t1)), two(coef, coef)), d[e], d[e + 1]);
            }
            if (!others)
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = 0.f;
            st_grad<T>(out, same, j + u * THREADS, sh.off, d);
        }
    }
    if (tid < 2) {
        const int p = tid ? sh.last : sh.first;
        if (p >= 0)
            for (int i = sh.begin(p); i < sh.end(p); ++i) out[i] = Vec<T>::from(grad(Vec<T>::to(z[i])));
    }
    __syncthreads();
    if (first && id >= from && id < to) {                              // the list's tokens
        float qs = 0.f;
        for (int k = tid; k < K; ++k) qs += ds.id[k] == id ? ds.q[k] : 0.f;
        out[id] = Vec<T>::from(none ? 0.f : g * (Q * ex2(max_nan(((zk - ref) * it - all) * LOG2E, FAR)) - qs));
    }
}

// ------------------------------------------------------------------ launches

// Blocks per row: enough that rows * C fill the device's block slots, but not less than one batch of loads per thread.
static int blocks_per_row(int rows, int vocab, int elem) {
    const int64_t bytes = (int64_t)vocab * elem;
    int C = 1;
    while (C < MAX_C && (int64_t)rows * C * 2 <= 4 * 148 && bytes / (2 * C) >= THREADS * 16) C *= 2;
    return C;
}

template <class A>
static cudaError_t launch(void (*k)(const A), const A &a, int rows, int C, size_t smem, cudaStream_t st) {
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)rows * (unsigned)C);
    c.blockDim = dim3(THREADS);
    c.dynamicSmemBytes = smem;
    c.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = C; at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    c.attrs = at;
    c.numAttrs = C > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&c, k, a);
}

static int elem_bytes(int dtype) { return dtype == PACER_F32 ? 4 : 2; }

cudaError_t logprobs(const Rows &r, const int32_t *tokens, const Window &win, const ScoreOut &out, cudaStream_t st) {
    const bool top = out.top > 0;
    ScoreArgs a{r, tokens, win, out, blocks_per_row(r.rows, r.vocab, elem_bytes(r.dtype))};
    const size_t smem = top ? sizeof(TopSlots) + (size_t)a.C * out.top * 8 : 0;
    auto go = [&](auto k0, auto k1) { return launch<ScoreArgs>(top ? k1 : k0, a, r.rows, a.C, smem, st); };
    if (r.dtype == PACER_F32) return go(k_logprobs<float, false>, k_logprobs<float, true>);
    if (r.dtype == PACER_BF16) return go(k_logprobs<__nv_bfloat16, false>, k_logprobs<__nv_bfloat16, true>);
    return go(k_logprobs<__half, false>, k_logprobs<__half, true>);
}

cudaError_t logprobs_backward(const Rows &r, const int32_t *tokens, const float *lse, const float *entropy, const float *g_logp,
                              const float *g_entropy, const float *g_lse, void *dz, int64_t ld_dz, cudaStream_t st) {
    BackArgs a{r, tokens, lse, entropy, g_logp, g_entropy, g_lse, dz, ld_dz, blocks_per_row(r.rows, r.vocab, elem_bytes(r.dtype))};
    auto go = [&](auto k0, auto k1) { return launch<BackArgs>(g_entropy ? k1 : k0, a, r.rows, a.C, 0, st); };
    if (r.dtype == PACER_F32) return go(k_logprobs_back<float, false>, k_logprobs_back<float, true>);
    if (r.dtype == PACER_BF16) return go(k_logprobs_back<__nv_bfloat16, false>, k_logprobs_back<__nv_bfloat16, true>);
    return go(k_logprobs_back<__half, false>, k_logprobs_back<__half, true>);
}

// A bit for each element of a block's share (at most three vectors more than an even one), and two words of slack.
static size_t mark_bytes(int vocab, int C) { return ((size_t)(vocab / C + 3 * 8) / 32 + 3) * 4; }

template <class T, int MODE>
static cudaError_t distill_any(const DistillArgs &a, cudaStream_t st) {
    const size_t marks = a.t.lse && MODE != GRAD ? mark_bytes(a.r.vocab, a.C) : 0;
    return launch<DistillArgs>(a.t.lse ? k_distill<T, true, MODE> : k_distill<T, false, MODE>, a, a.r.rows, a.C, marks, st);
}
template <int MODE>
static cudaError_t distill_type(DistillArgs &a, cudaStream_t st) {
    a.C = blocks_per_row(a.r.rows, a.r.vocab, elem_bytes(a.r.dtype));
    while (a.t.lse && mark_bytes(a.r.vocab, a.C) > 40 * 1024) a.C *= 2;      // (MAX_VOCAB / MAX_C bits fit)
    if (a.r.dtype == PACER_F32) return distill_any<float, MODE>(a, st);
    if (a.r.dtype == PACER_BF16) return distill_any<__nv_bfloat16, MODE>(a, st);
    return distill_any<__half, MODE>(a, st);
}

cudaError_t distill(const Rows &r, const Teacher &t, float *loss, float *lse, float *tail_lse, const float *weight, void *dz, int64_t ld_dz,
                    cudaStream_t st) {
    DistillArgs a{r, t, loss, lse, tail_lse, nullptr, nullptr, weight, dz, ld_dz, 1};
    return dz ? distill_type<LOSS_GRAD>(a, st) : distill_type<LOSS>(a, st);
}

cudaError_t distill_backward(const Rows &r, const Teacher &t, const float *lse, const float *tail_lse, const float *weight, void *dz,
                             int64_t ld_dz, cudaStream_t st) {
    DistillArgs a{r, t, nullptr, nullptr, nullptr, lse, tail_lse, weight, dz, ld_dz, 1};
    return distill_type<GRAD>(a, st);
}

}  // namespace lg

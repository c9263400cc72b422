// Gradients of the LM head fused with the scoring.  With z = hidden head^T (+ bias), p = exp(z - lse) and per row the incoming gradients,
//   dz = g_logp ([v = token] - p) + g_lse p - g_entropy p (log p + entropy),   dhidden = dz head,   dhead = dz^T hidden.
// z is computed again, and dz kept in bf16 for a piece of the vocabulary (all of it while that is at most 2 GB), as the operand of
// the two products: three products of 2 rows vocab d operations, bound by the tensor cores for many rows (8192 x 32 256 x 2048: 2.42 ms,
// 1.34 PFLOP/s, the rate that a long loop of library products holds under the power cap), by reading the head twice and writing dhead
// once for few.
//   k_head_z     z on tcgen05, dz by the epilogue
//   k_head_prod  both products in one launch: 256 x 256 tiles by pairs of blocks, operands by tensor copies as they lie in memory (dz is
//                read as its own transpose, hidden rows and head as MN-major operands: no transposed copies)
//   k_head_sum   dhidden from partial sums, where its product was cut along the vocabulary
// For the loss and its gradients in one call dz comes out of the loss's own pass (k_head_dz in head_score.cu): 2048 x 32 000 x 4096 1270 us, with
// z computed twice 1690.
// dz is rounded once, to bf16, as an operand has to be; sums are fp32.  1 - p of the row's token is -expm1(logp), off by what logp is: some 2^-24 of 1,
// of the f32 sum that it is the logarithm of.  (k_head_dz, which has the others' sum by itself, is off by that share of 1 - p.)
#include "head_grad.h"

#include <algorithm>
#include <type_traits>

#include "pair.cuh"
#include "two.cuh"

namespace hg {

using namespace fwd;
using namespace pr;
using namespace tw;

constexpr int TM = 128, TN = 256, PANEL = 64 * 128;        // rows of a block's half of a tile, columns of a tile; 64 rows x 64 columns
constexpr int STAGE = 4 * PANEL, STAGES = 5, OUT = 32 * 128, OUTS = 2;      // (a warp's output buffers)
constexpr int EPI_WARPS = 8, THREADS_G = 32 * (EPI_WARPS + 2), SMEM_Z = STAGE * STAGES + 1024, SMEM_P = SMEM_Z + EPI_WARPS * OUT * OUTS;
constexpr size_t MOST_DZ = (size_t)2 << 30;               // bytes of dz (without remainders) that are kept at a time
// The tensor cores truncate when they add to an accumulator.  Sums over more k blocks of 64 than these leave it every so often and are added in
// ordinary fp32, in the other accumulator's columns (LONG: one accumulator; a segment takes 100 times its addition).  With one accumulator for
// all of them dhead of rows whose terms have one sign was too small by 3e-5 for 8192 rows, 1.8e-3 for 300 000 and 6.5e-3 for a million.
constexpr int SEG_Z = 128, SEG_P = 256;
constexpr int FEW = 128;                                  // rows up to which dz comes with its rounding remainders
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct ZArgs {
    int32_t rows, width, v0, vocab, nkb, bn, mt, nt, a_rows, ld;   // v0: the piece's first token; ld: elements of a row of dz
    const int32_t *tokens, *bias_ids;
    float bias, sign;
    const float *logp, *lse, *entropy, *g_logp, *g_entropy, *g_lse;
    bf16 *dz, *low;                            // low: the rounding remainders, or NULL
};

struct PArgs {
    int32_t rows, width, d, dp, bn, nt;        // nt: tiles of d
    uint32_t by_nt;                            // 2^32 / nt, rounded up (exact quotients below 2^32 / nt)
    int32_t mt_w, mt_h, k_w, k_h, per, splits; // tiles of tokens and rows; k blocks of 64 of each product (of all planes), of a share of dhidden's
    int32_t n_h, n_w, early;                   // items of dhidden and dhead, dhead's that the less loaded workers take first
    int32_t add;                               // dhidden's sums are added to those that are there
    int32_t planes;                            // 2: dz and its remainders (at most 128 rows)
    // dhead by the threads' own stores, 32 bytes each, instead of copies out of shared memory: where a tile has more than a few k blocks they
    // run under the next tile's products and cost less (33 rows, 2 blocks: 32 us, by copies 26; 512 rows, 8: 26.1, 27.8; 2048, 32: 671, 679)
    int32_t direct;
    bf16 *dhead;
    int64_t ld_dhead;
    float *part;                               // [planes][splits][rows][dp], or NULL: dhidden is written
};

// The roles of a pair's blocks (warps 0..7 epilogue, 8 copies, 9 tensor cores) and what they share.
struct Pair {
    uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty[2];
    uint32_t tmem_slot;
    volatile int32_t gave_up;
};

__device__ __forceinline__ uint32_t pair_begin(Pair &s, int warp) {
    if (threadIdx.x == 0) {
        s.gave_up = 0;
        for (int i = 0; i < STAGES; ++i) { mbar_init(s.full + i, 1); mbar_init(s.empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(s.acc_full + i, 1); mbar_init(s.acc_empty + i, 2 * EPI_WARPS); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();                                                    // (both blocks' barriers are set up)
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("fence.proxy.async;" ::: "memory");                   // (what the kernels before wrote is read by the copy engine)
    return s.tmem_slot;
}
__device__ __forceinline__ void pair_end(uint32_t tmem, int warp) {
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync();                                                    // (nothing of one block is in use by the other)
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}
// Waits until none of the n copies issued is in flight (a pair's arrive at its first block's barriers; the second ends after it).
__device__ __forceinline__ void drain(Pair &s, int n, int rank) {
    for (int j = max(0, n - STAGES); j < n && rank == 0; ++j)
        for (unsigned it = 0; it < MBAR_SPIN_LIMIT && !mbar_try_wait(s.full + j % STAGES, ((uint32_t)(j / STAGES)) & 1u); ++it) {}
}
// k blocks that are worked on meanwhile: a tile's sums over a million rows or tokens take milliseconds.  (An empty share's may be below 0: one of 4
// shares of the last 283 of 2 093 339 tokens.)
__host__ __device__ constexpr unsigned wait_limit(int blocks) { return MBAR_SPIN_LIMIT * (1u + (unsigned)(blocks > 0 ? blocks : 0) / 1024u); }
static_assert(wait_limit(-1) == MBAR_SPIN_LIMIT && wait_limit(-64) == MBAR_SPIN_LIMIT && wait_limit(1023) == MBAR_SPIN_LIMIT, "the usual wait");
static_assert(wait_limit(1 << 15) == 33 * MBAR_SPIN_LIMIT, "2^21 tokens or rows");
__device__ __forceinline__ bool all_wait(Pair &s, uint64_t *bar, uint32_t parity, int blocks = 0) {
    return __all_sync(0xffffffffu, wait_h(&s.gave_up, bar, parity, wait_limit(blocks)));
}
__device__ __forceinline__ uint32_t pair_idesc(int n) { return (umma_idesc(n) & ~(31u << 24)) | (256u >> 4) << 24; }
// An MN-major operand in the 128-byte swizzle: rows (k) of 64 channels, eight of them 1 KB, the next 64 channels a panel further.
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFF) | ((uint64_t)(PANEL >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// The i-th accumulator: which of the two, and the parity of its barriers' phase.
template <bool LONG> __device__ __forceinline__ int which(int i) { return LONG ? 0 : i & 1; }
template <bool LONG> __device__ __forceinline__ uint32_t phase(int i) { return (uint32_t)(LONG ? i : i >> 1) & 1u; }
template <bool LONG> __device__ __forceinline__ void release_acc(Pair &s, int i, int lane) {
    tc_fence_before();
    __syncwarp();
    if (lane == 0) acc_release(s.acc_empty + which<LONG>(i));
}
// sum (tensor memory, of the segments before; the first sets it) += acc, 32 columns.
__device__ __forceinline__ void add_segment(uint32_t sum, uint32_t acc, bool first) {
    uint32_t v[32], w[32];
    tmem_ld32(acc, v);
    if (!first) {
        tmem_ld32(sum, w);
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(w[e]) + __uint_as_float(v[e]));
    }
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,"
                 "%28,%29,%30,%31,%32};"
                 ::"r"(sum), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
                   "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]),
                   "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
// ----------------------------------------------------------------------------- dz of a piece of the vocabulary

// Persistent as k_head_score: row tiles vary fastest.
template <bool LONG>
__global__ void __launch_bounds__(THREADS_G, 1) k_head_z(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const ZArgs a) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ Pair s;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    unsigned char *smem = smem_raw + (-(int)smem_u32(smem_raw) & 1023);      // (the same in both blocks)
    const int rank = blockIdx.x & 1, worker = blockIdx.x >> 1, workers = gridDim.x >> 1, tiles = a.mt * a.nt;
    const uint32_t tmem = pair_begin(s, warp);

    if (warp == 8) {
        uint64_t policy;                                               // lane 0 hidden rows, lane 1 the head
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
        if (lane == 0) asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(policy));
        const uint32_t full0 = first_block(s.full);
        int n = 0;
        bool ok = true;
        for (int t = worker; t < tiles && ok; t += workers) {
            const int y = lane ? (t / a.mt) * a.bn + rank * (a.bn >> 1) : (t % a.mt) * (2 * TM) + rank * TM;
            for (int kb = 0; kb < a.nkb; ++kb, ++n) {
                const int slot = n % STAGES;
                ok = all_wait(s, s.empty + slot, (((uint32_t)(n / STAGES)) & 1u) ^ 1u);
                if (!ok) break;
                if (lane == 0 && rank == 0) mbar_expect_tx(s.full + slot, (uint32_t)(2 * a.a_rows + a.bn) * 128u);   // (both blocks' bytes)
                if (lane < 2) tma_2d<true>(smem + slot * STAGE + lane * 2 * PANEL, lane ? &map_b : &map_a, kb * 64, y, full0 + slot * 8, policy);
            }
        }
        if (lane == 0) drain(s, n, rank);
    } else if (warp == 9) {
        const uint32_t on = elect_lane(), idesc = pair_idesc(a.bn);        // (all lanes wait, one of the first block issues)
        int n = 0, i = 0;
        bool ok = true;
        for (int t = worker; t < tiles && ok && rank == 0; t += workers, ++i) {
            ok = all_wait(s, s.acc_empty + which<LONG>(i), phase<LONG>(i) ^ 1u);
            if (!ok) break;
            const uint32_t acc = tmem + which<LONG>(i) * 256u;
            for (int kb = 0; kb < a.nkb; ++kb, ++n) {
                if (LONG && kb && kb % SEG_Z == 0) {
                    umma2_commit_if(on, s.acc_full + which<LONG>(i));
                    ++i;
                    ok = all_wait(s, s.acc_empty + which<LONG>(i), phase<LONG>(i) ^ 1u);
                    if (!ok) break;
                }
                const int slot = n % STAGES;
                ok = all_wait(s, s.full + slot, ((uint32_t)(n / STAGES)) & 1u);
                if (!ok) break;
                tc_fence_after();
                const uint32_t a0 = smem_u32(smem + slot * STAGE), b0 = a0 + 2 * PANEL;
#pragma unroll
                for (int k16 = 0; k16 < 4; ++k16)
                    umma2_if(on, acc, umma_desc(a0 + k16 * 32), umma_desc(b0 + k16 * 32), idesc, (LONG ? kb % SEG_Z : kb) > 0 || k16 > 0 ? 1u : 0u);
                umma2_commit_if(on, s.empty + slot);
            }
            if (ok) umma2_commit_if(on, s.acc_full + which<LONG>(i));
        }
    } else {
        const int quad = warp & 3, half = warp >> 2;
        const int chunks = a.bn >> 5, c0 = half ? (chunks + 1) >> 1 : 0, c1 = half ? chunks : (chunks + 1) >> 1;
        int i = 0;
        bool ok = true;                                                // (once a wait has given up, the tiles left become NaN)
        for (int t = worker; t < tiles; t += workers, ++i) {
            const int n0 = (t / a.mt) * a.bn, r = (t % a.mt) * (2 * TM) + rank * TM + quad * 32 + lane;
            const bool live = r < a.rows;
            // dz = p (c + h log p), with `at` in the token's place
            float gl = 0.f, c = 0.f, h = 0.f, lse = 0.f, lp = 0.f;
            int tok = -1, bid = -1;
            if (live) {
                const int id = a.tokens ? a.tokens[r] : -1;
                if (id >= 0 && id < a.vocab && a.g_logp) {
                    gl = a.sign * a.g_logp[r];
                    lp = a.logp[r];
                    tok = id - a.v0 - n0;
                }
                if (a.bias_ids) bid = a.bias_ids[r] - a.v0 - n0;
                lse = a.lse[r] * LOG2E;
                c = (a.g_lse ? a.g_lse[r] : 0.f) - gl;
                if (a.g_entropy) { const float e = a.g_entropy[r]; c = fmaf(-e, a.entropy[r], c); h = -e * LN2; }
            }
            uint32_t acc = tmem + which<LONG>(i) * 256u + ((uint32_t)(quad * 32) << 16);
            if (LONG) {
                for (int kb = 0;; ++i) {
                    if (ok) ok = all_wait(s, s.acc_full + which<LONG>(i), phase<LONG>(i));
                    tc_fence_after();
                    for (int k = c0; k < c1 && ok; ++k) add_segment(acc + 256u + k * 32, acc + k * 32, kb == 0);
                    release_acc<LONG>(s, i, lane);
                    if ((kb += SEG_Z) >= a.nkb) break;
                }
                acc += 256u;
            } else {
                if (ok) ok = all_wait(s, s.acc_full + which<LONG>(i), phase<LONG>(i));
                tc_fence_after();
            }
            for (int k = c0; k < c1; ++k) {
                const int at = k * 32;
                if (n0 + at >= a.ld) break;
                uint32_t v[32];
                tmem_ld32(acc + at, v);
                if ((uint32_t)(bid - at) < 32u)
#pragma unroll
                    for (int e = 0; e < 32; ++e) {                     // (no lower than -1e30: 2^t is 0, and t finite)
                        const float z = __uint_as_float(v[e]) + a.bias;
                        v[e] = bid - at == e ? __float_as_uint(z < -1e30f ? -1e30f : z) : v[e];
                    }
                uint32_t w[16], l16[16];
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const Two l = fma2(two(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), two(LOG2E, LOG2E), two(-lse, -lse));
                    float l0, l1, g0, g1;
                    apart(l, l0, l1);
                    apart(mul2(two(ex2(l0), ex2(l1)), fma2(two(h, h), l, two(c, c))), g0, g1);
                    w[e >> 1] = pack(g0, g1);
                    if (a.low) l16[e >> 1] = pack(g0 - __uint_as_float(w[e >> 1] << 16), g1 - __uint_as_float(w[e >> 1] & 0xffff0000u));
                }
                if (!ok)
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = 0x7fff7fffu;
                if (live) {
                    bf16 *p = a.dz + (size_t)r * a.ld + n0 + at, *q = a.low + (size_t)r * a.ld + n0 + at;
                    st32(p, w);
                    st32(p + 16, w + 8);
                    if (a.low) {
                        st32(q, l16);
                        st32(q + 16, l16 + 8);
                    }
                    if ((uint32_t)(tok - at) < 32u && ok) {                // the token's own
                        float z = 0.f;
#pragma unroll
                        for (int e = 0; e < 32; ++e) z = tok - at == e ? __uint_as_float(v[e]) : z;
                        const float l = fmaf(z, LOG2E, -lse), x = ex2(l) * fmaf(h, l, c + gl) - gl * expm1f(lp);
                        p[tok - at] = __float2bfloat16_rn(x);
                        if (a.low) q[tok - at] = __float2bfloat16_rn(x - __bfloat162float(__float2bfloat16_rn(x)));
                    }
                }
            }
            if (!LONG) release_acc<LONG>(s, i, lane);
        }
    }
    pair_end(tmem, warp);
}

// ----------------------------------------------------------------------------- the products

struct Item { int32_t to_head, m0, n0, k0, k1, split; };
// A worker's items one after another.  dhidden's long ones are dealt out first; where they do not come out even, the workers with one less take
// `early` rounds of dhead's before the others join.
struct Walk {
    int t, left, next, early, less, workers, base;
    __device__ __forceinline__ Walk(const PArgs &a, int worker, int n_workers) {
        workers = n_workers;
        const int rem = a.n_h % workers;
        left = a.n_h / workers + (worker < rem);
        t = worker;
        const bool fewer = rem && worker >= rem;
        less = workers - rem;
        early = fewer ? a.early : 0;
        base = rem ? a.early * less : 0;       // dhead's first tile that all workers take part in
        next = fewer ? worker - rem : base + worker;
        if (fewer && !early) next = base + worker;
        base += worker;
    }
    __device__ __forceinline__ bool operator()(const PArgs &a, Item &it) {
        if (left) {
            --left;
            const int n = t % a.nt, q = t / a.nt, m = q % a.mt_h;
            it.split = q / a.mt_h;
            it.to_head = 0; it.m0 = m * 2 * TM; it.n0 = n * a.bn; it.k0 = it.split * a.per; it.k1 = min(a.k_h, it.k0 + a.per);
            t += workers;
            return true;
        }
        if (next >= a.n_w) return false;
        const int m = a.nt > 1 ? (int)__umulhi((uint32_t)next, a.by_nt) : next;       // next / nt
        it.to_head = 1; it.m0 = m * 2 * TM; it.n0 = (next - m * a.nt) * a.bn; it.k0 = 0; it.k1 = a.k_w; it.split = 0;
        if (early && --early == 0) next = base;
        else next += early ? less : workers;
        return true;
    }
};

// dhead tiles: A = dz by its columns (MN-major), B = hidden (MN-major), k = rows.  dhidden tiles: A = dz (K-major), B = head (MN-major),
// k = tokens.  All tensor copies are 64 x 64: a panel of an MN-major operand, half of a K-major one.
// Up to 128 rows dz comes with its rounding remainders, which cost little there: dhead has twice the k blocks, which its stores outlast, and the
// second block of a pair, whose rows would be empty, multiplies the remainders (its sums are a share of their own).
template <bool LONG>
__global__ void __launch_bounds__(THREADS_G, 1) k_head_prod(const __grid_constant__ CUtensorMap map_z, const __grid_constant__ CUtensorMap map_low,
                                                            const __grid_constant__ CUtensorMap map_x,
                                                            const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_dw,
                                                            const __grid_constant__ CUtensorMap map_dx, const PArgs a) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    __shared__ Pair s;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    unsigned char *smem = smem_raw + (-(int)smem_u32(smem_raw) & 1023);
    const int rank = blockIdx.x & 1, worker = blockIdx.x >> 1, workers = gridDim.x >> 1, half_n = a.bn >> 1;
    const uint32_t tmem = pair_begin(s, warp);
    Walk walk(a, worker, workers);
    Item it;

    if (warp == 8) {
        // lanes 0, 1 the panels of A, lanes 2, 3 those of B, all four by one instruction: by one lane, with the kind looked up per copy, the copies
        // did not keep up with the products (2048 x 32 000 x 4096: 750 us, with a loop for each kind 706)
        const int q = lane & 1;
        const bool copies = lane < 2 || (lane < 4 && q * 64 < half_n);
        uint64_t normal;
        asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(normal));
        const uint32_t full0 = first_block(s.full);
        int n = 0;
        bool ok = true;
        while (ok && walk(a, it)) {
            const int m = it.m0 + (it.to_head || a.planes == 1 ? rank * TM : 0) + q * 64, nb = it.n0 + rank * half_n + q * 64;
            const bool moves = !it.to_head && lane < 2;               // (k along the operand's rows)
            const int dx = moves ? 64 : 0, dy = 64 - dx, planes = it.to_head ? a.planes : 1, k1 = it.to_head ? a.k_w / a.planes : it.k1;
            for (int plane = 0; plane < planes && ok; ++plane) {
                const bool low = it.to_head ? plane : a.planes == 2 && rank;
                const CUtensorMap *map = lane < 2 ? low ? &map_low : &map_z : it.to_head ? &map_x : &map_w;
                int x = lane < 2 ? moves ? it.k0 * 64 : m : nb, y = moves ? m : it.k0 * 64;
                for (int kb = it.k0; kb < k1; ++kb, ++n) {
                    const int slot = n % STAGES;
                    ok = all_wait(s, s.empty + slot, (((uint32_t)(n / STAGES)) & 1u) ^ 1u);
                    if (!ok) break;
                    if (lane == 0 && rank == 0) mbar_expect_tx(s.full + slot, (uint32_t)(2 * TM + a.bn) * 128u);
                    if (copies) tma_2d<true>(smem + slot * STAGE + lane * PANEL, map, x, y, full0 + slot * 8, normal);
                    x += dx;
                    y += dy;
                }
            }
        }
        if (lane == 0) drain(s, n, rank);
    } else if (warp == 9) {
        const uint32_t on = elect_lane(), idesc = pair_idesc(a.bn) | (1u << 16);
        int n = 0;
        bool ok = true;
        // (a loop for each kind: with the kind looked up per product the descriptors left the uniform registers, 717 -> 759 us in all)
        const auto multiply = [&](auto kind, uint32_t acc, int blocks) {
            constexpr bool to_head = decltype(kind)::value;
            for (int kb = 0; kb < blocks; ++kb, ++n) {
                const int slot = n % STAGES;
                ok = all_wait(s, s.full + slot, ((uint32_t)(n / STAGES)) & 1u);
                if (!ok) break;
                tc_fence_after();
                const uint32_t a0 = smem_u32(smem + slot * STAGE), b0 = a0 + 2 * PANEL;
#pragma unroll
                for (int k16 = 0; k16 < 4; ++k16)
                    umma2_if(on, acc, to_head ? desc_mn(a0 + k16 * 2048) : umma_desc(a0 + k16 * 32), desc_mn(b0 + k16 * 2048),
                             to_head ? idesc | (1u << 15) : idesc, kb > 0 || k16 > 0 ? 1u : 0u);
                umma2_commit_if(on, s.empty + slot);
            }
        };
        for (int j = 0; ok && rank == 0 && walk(a, it);) {
            int left = it.to_head ? a.k_w : it.k1 - it.k0;
            do {                                                       // (a segment; an empty share has one of no blocks)
                ok = all_wait(s, s.acc_empty + which<LONG>(j), phase<LONG>(j) ^ 1u);
                if (!ok) break;
                const uint32_t acc = tmem + which<LONG>(j) * 256u;
                const int blocks = LONG ? min(left, SEG_P) : left;
                if (it.to_head) multiply(std::true_type{}, acc, blocks);
                else multiply(std::false_type{}, acc, blocks);
                if (ok) umma2_commit_if(on, s.acc_full + which<LONG>(j));
                ++j;
                left -= blocks;
            } while (LONG && ok && left > 0);
        }
    } else {
        const int quad = warp & 3, half = warp >> 2;
        unsigned char *outs = smem + STAGES * STAGE + warp * OUT * OUTS;
        int stored = 0;
        bool ok = true;
        for (int j = 0; walk(a, it); ++j) {
            uint32_t acc = tmem + which<LONG>(j) * 256u + ((uint32_t)(quad * 32) << 16) + half * half_n;
            if (LONG) {
                for (int k = it.k0;; ++j) {
                    if (ok) ok = all_wait(s, s.acc_full + which<LONG>(j), phase<LONG>(j), SEG_P);
                    tc_fence_after();
                    for (int c = 0; c < half_n && ok; c += 32) add_segment(acc + 256u + c, acc + c, k == it.k0);
                    release_acc<LONG>(s, j, lane);
                    if ((k += SEG_P) >= it.k1) break;
                }
                acc += 256u;
            } else {
                if (ok) ok = all_wait(s, s.acc_full + which<LONG>(j), phase<LONG>(j), it.k1 - it.k0);
                tc_fence_after();
            }
            const int plane = !it.to_head && a.planes == 2 ? rank : 0;
            const int m = it.m0 + (plane ? 0 : rank * TM) + quad * 32, n0 = it.n0 + half * half_n, last = it.to_head ? a.width : a.rows;
            const bool sums = !it.to_head && a.part;
            for (int c = 0; c < half_n; c += 64) {
                if (m >= last || n0 + c >= a.dp) break;
                uint32_t v[64];
                tmem_ld32(acc + c, *reinterpret_cast<uint32_t(*)[32]>(v));
                tmem_ld32(acc + c + 32, *reinterpret_cast<uint32_t(*)[32]>(v + 32));
                if (!ok || it.k0 >= it.k1)                             // (a share of the last, narrower piece may be empty)
#pragma unroll
                    for (int e = 0; e < 64; ++e) v[e] = ok ? 0u : 0x7fffffffu;
                if (sums) {
                    if (m + lane < last) {
                        float *p = a.part + ((size_t)(plane * a.splits + it.split) * a.rows + m + lane) * a.dp + n0 + c;
#pragma unroll
                        for (int e = 0; e < 64; e += 8) {
                            if (a.add) {
                                const float4 x = *reinterpret_cast<const float4 *>(p + e), y = *reinterpret_cast<const float4 *>(p + e + 4);
                                const float o[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
                                for (int f = 0; f < 8; ++f) v[e + f] = __float_as_uint(__uint_as_float(v[e + f]) + o[f]);
                            }
                            st32(p + e, v + e);
                        }
                    }
                    continue;
                }
                if (it.to_head && a.direct) {
                    if (m + lane < last) {
                        bf16 *p = a.dhead + (size_t)(m + lane) * a.ld_dhead + n0 + c;
#pragma unroll
                        for (int e = 0; e < 64; e += 16) {
                            uint32_t w[8];
#pragma unroll
                            for (int f = 0; f < 8; ++f) w[f] = pack(__uint_as_float(v[e + 2 * f]), __uint_as_float(v[e + 2 * f + 1]));
                            if (n0 + c + e < a.d) st32(p + e, w);
                        }
                    }
                    continue;
                }
                unsigned char *out = outs + (stored++ % OUTS) * OUT;
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(OUTS - 1) : "memory");   // (its last copy has left)
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const uint32_t *u = v + 8 * q;
                    *reinterpret_cast<uint4 *>(out + lane * 128 + ((q ^ (lane & 7)) << 4)) =
                        make_uint4(pack(__uint_as_float(u[0]), __uint_as_float(u[1])), pack(__uint_as_float(u[2]), __uint_as_float(u[3])),
                                   pack(__uint_as_float(u[4]), __uint_as_float(u[5])), pack(__uint_as_float(u[6]), __uint_as_float(u[7])));
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    const CUtensorMap *mo = it.to_head ? &map_dw : &map_dx;
                    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(mo), "r"(n0 + c), "r"(m),
                                 "r"(smem_u32(out)) : "memory");
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                }
            }
            if (!LONG) release_acc<LONG>(s, j, lane);
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    pair_end(tmem, warp);
}

// dhidden = the sum of the shares: four lanes, 8 apart, for eight columns, each a quarter of the shares.
__global__ void __launch_bounds__(256) k_head_sum(const float *part, int splits, int rows, int d, int dp, bf16 *out, int64_t ld) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int per = d >> 3, q = (threadIdx.x >> 3) & 3;
    const int64_t i = (int64_t)blockIdx.x * 64 + (threadIdx.x >> 5) * 8 + (threadIdx.x & 7);
    const bool on = i < (int64_t)rows * per;
    const int64_t r = on ? i / per : 0, c = on ? (i - r * per) * 8 : 0;
    float v[8] = {};
#pragma unroll 4
    for (int k = on ? q : splits; k < splits; k += 4) {
        const float4 *p = reinterpret_cast<const float4 *>(part + ((size_t)k * rows + r) * dp + c);
        const float4 x = __ldcg(p), y = __ldcg(p + 1);
        v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w; v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] += __shfl_xor_sync(~0u, v[e], 8);
        v[e] += __shfl_xor_sync(~0u, v[e], 16);
    }
    if (on && q == 0) *reinterpret_cast<uint4 *>(out + r * ld + c) = make_uint4(pack(v[0], v[1]), pack(v[2], v[3]), pack(v[4], v[5]), pack(v[6], v[7]));
}

// ----------------------------------------------------------------------------- host

struct Plan {
    int pieces, width;                     // tokens of a piece
    int ld;                                // of dz
    int bn, nt, dp, mt_h, splits, per, planes;
    size_t plane_bytes, part_bytes;
    size_t bytes() const { return plane_bytes * planes + part_bytes; }
};
static int up(int64_t a, int b) { return (int)((a + b - 1) / b); }

// A unit of time is a k block of a tile, 512 cycles.  A tile's epilogue and start count as four.
constexpr int EXTRA = 4;
static Plan plan_of(int rows, int vocab, int d, bool to_hidden, bool to_head, int n_sm) {
    Plan p;
    const int64_t most = std::max<int64_t>(256, (int64_t)(MOST_DZ / 2 / (size_t)rows) / 256 * 256);
    p.pieces = up(vocab, (int)std::min<int64_t>(most, 1 << 24));
    p.width = p.pieces == 1 ? vocab : up(up(vocab, p.pieces), 256) * 256;
    p.pieces = up(vocab, p.width);
    p.ld = up(p.width, 64) * 64;
    p.bn = d <= 128 ? 128 : 256;
    p.nt = up(d, p.bn);
    p.dp = up(d, 64) * 64;
    p.mt_h = up(rows, 2 * TM);
    p.planes = rows <= FEW ? 2 : 1;
    const int workers = n_sm / 2, k_h = up(p.width, 64);
    // dhidden's product is cut along the tokens into the number of shares with the least time until the last worker is done
    const int64_t tiles = (int64_t)p.mt_h * p.nt, head = to_head ? (int64_t)up(p.width, 2 * TM) * p.nt * (up(rows, 64) * p.planes + EXTRA) : 0;
    p.splits = 1;
    p.per = k_h;
    if (to_hidden) {
        double best = 0;
        for (int n = 1; n <= 64 && n <= k_h; ++n) {
            const int per = up(k_h, n), shares = up(k_h, per);
            const double own = (double)up(tiles * shares, workers) * (per + EXTRA), all = ((double)tiles * shares * (per + EXTRA) + head) / workers;
            // (sums written and read at 6 TB/s; a launch)
            const double cost = std::max(own, all) + (shares > 1 || p.pieces > 1 || p.planes > 1 ? 10 + (double)shares * p.planes * rows * p.dp * 8 / 1.6e6 : 0);
            if (n == 1 || cost < best) { best = cost; p.splits = shares; p.per = per; }
        }
    }
    p.plane_bytes = ((size_t)rows * p.ld * 2 + 255) & ~(size_t)255;
    p.part_bytes = to_hidden && (p.splits > 1 || p.pieces > 1 || p.planes > 1) ? (size_t)p.planes * p.splits * rows * p.dp * 4 : 0;
    return p;
}

size_t scratch_bytes(int rows, int vocab, int d, int n_sm) {
    size_t most = 0;
    for (int k = 1; k < 4; ++k) {
        const Plan p = plan_of(rows, vocab, d, k & 1, k & 2, n_sm);
        most = std::max(most, p.bytes());
    }
    return most;
}

static cudaError_t opt_in() {              // (per device)
    static bool done[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev >= 0 && dev < 64 && done[dev])) return e;
    e = cudaFuncSetAttribute(k_head_z<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_Z);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_head_z<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_Z);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_head_prod<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_P);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_head_prod<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_P);
    if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
    return e;
}

// A launch that waits by itself for the kernel before it (early: it may be set up while that runs).
struct Launch {
    cudaLaunchConfig_t c = {};
    cudaLaunchAttribute at[2];
    Launch(unsigned grid, unsigned threads, size_t smem, cudaStream_t st, bool pair, bool early) {
        c.gridDim = dim3(grid);
        c.blockDim = dim3(threads);
        c.dynamicSmemBytes = smem;
        c.stream = st;
        c.attrs = at;
        if (early) {
            at[c.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            at[c.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
        }
        if (pair) {
            at[c.numAttrs].id = cudaLaunchAttributeClusterDimension;
            at[c.numAttrs].val.clusterDim.x = 2;
            at[c.numAttrs].val.clusterDim.y = at[c.numAttrs].val.clusterDim.z = 1;
            ++c.numAttrs;
        }
    }
};

// Tokens of a tile of z: the width with the least waves x (width + 16).
static int z_width(int mt, int width, int workers) {
    int best = TN;
    int64_t best_cost = INT64_MAX;
    for (int w = TN; w >= 32; w -= 32) {
        const int64_t tiles = (int64_t)mt * up(width, w), cost = (tiles + workers - 1) / workers * (w + 16);
        if (cost < best_cost) { best_cost = cost; best = w; }
    }
    return best;
}

// The products of dz of one piece, and after the last one the sum.
static cudaError_t products(const Args &a, const Plan &p, EncodeFn encode, int piece, bf16 *dz, bf16 *low, float *part, int workers, cudaStream_t st, bool *no_maps) {
    const int v0 = piece * p.width, width = std::min(p.width, a.vocab - v0);
    const bf16 *head = reinterpret_cast<const bf16 *>(a.head) + (size_t)v0 * a.ld_head;
    bf16 *dhead = a.dhead ? reinterpret_cast<bf16 *>(a.dhead) + (size_t)v0 * a.ld_dhead : nullptr;
    CUtensorMap mz, ml, mx, mw, mdw, mdx;
    if (!make_map(encode, &mz, dz, p.ld, a.rows, width, 64) || (low && !make_map(encode, &ml, low, p.ld, a.rows, width, 64)) ||
        !make_map(encode, &mx, a.hidden, a.ld_hidden, a.rows, a.d, 64) || !make_map(encode, &mw, head, a.ld_head, width, a.d, 64) ||
        (dhead && !make_map(encode, &mdw, dhead, a.ld_dhead, width, a.d, 32)) ||
        (a.dhidden && !part && !make_map(encode, &mdx, a.dhidden, a.ld_dhidden, a.rows, a.d, 32))) {
        *no_maps = true;
        return cudaSuccess;
    }
    if (!low) ml = mz;                     // (what is not used)
    if (!dhead) mdw = mw;
    if (!a.dhidden || part) mdx = mw;
    PArgs q;
    q.rows = a.rows; q.width = width; q.d = a.d; q.dp = p.dp; q.bn = p.bn; q.nt = p.nt;
    q.by_nt = (uint32_t)(((uint64_t)1 << 32) / p.nt + (p.nt & (p.nt - 1) ? 1 : 0));
    q.mt_w = up(width, 2 * TM); q.mt_h = p.mt_h; q.planes = p.planes; q.k_w = up(a.rows, 64) * p.planes; q.k_h = up(width, 64);
    q.splits = p.splits; q.per = up(q.k_h, p.splits);
    q.n_h = a.dhidden ? p.splits * p.mt_h * p.nt : 0;
    q.n_w = dhead ? q.mt_w * p.nt : 0;
    q.early = (q.per + EXTRA) / (q.k_w + EXTRA);
    q.add = piece > 0;
    q.part = part; q.dhead = dhead; q.ld_dhead = a.ld_dhead;
    q.direct = q.k_w >= 4 && a.d % 16 == 0 && (((uintptr_t)dhead | (uintptr_t)(a.ld_dhead * 2)) & 31) == 0;
    Launch l((unsigned)std::min<int64_t>(workers, (int64_t)q.n_h + q.n_w) * 2, THREADS_G, SMEM_P, st, true, true);
    const bool segments = (dhead && q.k_w > SEG_P) || (a.dhidden && q.per > SEG_P);
    cudaError_t e = segments ? cudaLaunchKernelEx(&l.c, k_head_prod<true>, mz, ml, mx, mw, mdw, mdx, q) : cudaLaunchKernelEx(&l.c, k_head_prod<false>, mz, ml, mx, mw, mdw, mdx, q);
    if (e != cudaSuccess || !part || piece < p.pieces - 1) return e;
    Launch s((unsigned)(((int64_t)a.rows * (a.d >> 3) + 63) / 64), 256, 0, st, false, true);
    return cudaLaunchKernelEx(&s.c, k_head_sum, (const float *)part, p.splits * p.planes, a.rows, a.d, p.dp, reinterpret_cast<bf16 *>(a.dhidden), a.ld_dhidden);
}

struct Places { bf16 *dz, *low; float *part; };
static Places places(const Plan &p, void *scratch) {
    char *at = reinterpret_cast<char *>(scratch);
    return {reinterpret_cast<bf16 *>(at), p.planes == 2 ? reinterpret_cast<bf16 *>(at + p.plane_bytes) : nullptr,
            p.part_bytes ? reinterpret_cast<float *>(at + p.plane_bytes * p.planes) : nullptr};
}

cudaError_t run(const Args &a, void *scratch, int n_sm, bool after, cudaStream_t st, bool *no_maps) {
    *no_maps = false;
    EncodeFn encode;
    cudaError_t e = encode_fn(&encode);
    if (e != cudaSuccess) return e;
    if (!encode) { *no_maps = true; return cudaSuccess; }
    e = opt_in();
    if (e != cudaSuccess) return e;
    const Plan p = plan_of(a.rows, a.vocab, a.d, a.dhidden, a.dhead, n_sm);
    const int workers = n_sm / 2;
    const Places at = places(p, scratch);
    for (int i = 0; i < p.pieces; ++i) {
        ZArgs z;
        z.v0 = i * p.width; z.width = std::min(p.width, a.vocab - z.v0);
        z.rows = a.rows; z.vocab = a.vocab; z.nkb = up(a.d, 64); z.mt = up(a.rows, 2 * TM); z.ld = p.ld;
        z.bn = z_width(z.mt, z.width, workers);
        z.nt = up(z.width, z.bn);
        z.a_rows = std::min(TM, (a.rows + 7) & ~7);
        z.tokens = a.tokens; z.bias_ids = a.bias_ids; z.bias = a.bias; z.sign = a.sign;
        z.logp = a.logp; z.lse = a.lse; z.entropy = a.entropy; z.g_logp = a.g_logp; z.g_entropy = a.g_entropy; z.g_lse = a.g_lse;
        z.dz = at.dz; z.low = at.low;
        CUtensorMap ma, mb;
        if (!make_map(encode, &ma, a.hidden, a.ld_hidden, a.rows, a.d, z.a_rows) ||
            !make_map(encode, &mb, reinterpret_cast<const bf16 *>(a.head) + (size_t)z.v0 * a.ld_head, a.ld_head, z.width, a.d, z.bn / 2)) {
            *no_maps = true;
            return cudaSuccess;
        }
        Launch l((unsigned)std::min<int64_t>(workers, (int64_t)z.mt * z.nt) * 2, THREADS_G, SMEM_Z, st, true, after || i);
        e = z.nkb > SEG_Z ? cudaLaunchKernelEx(&l.c, k_head_z<true>, ma, mb, z) : cudaLaunchKernelEx(&l.c, k_head_z<false>, ma, mb, z);
        if (e == cudaSuccess) e = products(a, p, encode, i, at.dz, at.low, at.part, workers, st, no_maps);
        if (e != cudaSuccess || *no_maps) return e;
    }
    return cudaSuccess;
}

// Where dz of the whole vocabulary is kept the loss's pass leaves it (hs::Args::dz), else z is computed again piece by piece.  The loss's own scratch
// lies behind dz in the first case; in the second it is free again when dz is written, and shares its memory.
static size_t rows_bytes(int rows) { return ((size_t)rows * 8 + 255) & ~(size_t)255; }

size_t nll_scratch_bytes(int rows, int vocab, int d, int n_sm) {
    const size_t own = (hs::scratch_bytes(rows, vocab) + 255) & ~(size_t)255, most = scratch_bytes(rows, vocab, d, n_sm);
    return plan_of(rows, vocab, d, true, true, n_sm).pieces == 1 ? own + most : rows_bytes(rows) + std::max(own, most);
}

cudaError_t run_nll(const Args &a, float *loss, void *scratch, int n_sm, cudaStream_t st, bool *no_maps) {
    const Plan p = plan_of(a.rows, a.vocab, a.d, a.dhidden, a.dhead, n_sm);
    const bool grads = a.dhidden || a.dhead;
    hs::Args h = {a.hidden, a.head, a.ld_hidden, a.ld_head, a.rows, a.vocab, a.d, a.tokens, a.bias_ids, a.bias, nullptr, nullptr, nullptr};
    h.loss = loss;
    if (grads && p.pieces == 1) {
        const size_t own = (hs::scratch_bytes(a.rows, a.vocab) + 255) & ~(size_t)255;
        const Places at = places(p, reinterpret_cast<char *>(scratch) + own);
        h.dz = at.dz; h.dz_low = at.low; h.ld_dz = p.ld; h.weight = a.g_logp;
        cudaError_t e = hs::run(h, scratch, n_sm, st, no_maps);
        if (e != cudaSuccess || *no_maps) return e;
        EncodeFn encode;
        e = encode_fn(&encode);
        if (e == cudaSuccess) e = opt_in();
        return e != cudaSuccess ? e : products(a, p, encode, 0, at.dz, at.low, at.part, n_sm / 2, st, no_maps);
    }
    float *logp = reinterpret_cast<float *>(scratch), *lse = logp + a.rows;
    void *rest = reinterpret_cast<char *>(scratch) + rows_bytes(a.rows);
    h.logp = logp; h.lse = lse;
    cudaError_t e = hs::run(h, rest, n_sm, st, no_maps);
    if (e != cudaSuccess || *no_maps || !grads) return e;
    Args b = a;
    b.logp = logp;
    b.lse = lse;
    return run(b, rest, n_sm, true, st, no_maps);
}

}  // namespace hg

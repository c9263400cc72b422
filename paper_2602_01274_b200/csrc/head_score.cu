// LM head fused with the scoring of given tokens: z = hidden head^T, and of each row of z only its log-sum-exp, its entropy and
// the logit of one token.  The logits are never written: [rows][vocab] f32 would be 262 MB for 2048 rows of 32 000.  (For the loss's gradients,
// KEEP below, each share of a half tile's largest is, in 16 bits.)
//
// Many rows are bound by the tensor cores (2 rows vocab d operations), few by reading the head once.  One kernel does both: tiles
// of 128 rows (256 by a pair of blocks) x up to 256 tokens on tcgen05, operands by tensor copies in the 128-byte swizzle, 192 KB of
// stages, two accumulators so that a tile's epilogue runs under the next tile's products.  With few rows the 128-row operand is
// mostly unused, but the tensor cores are not what bounds: a 256-token tile takes 128 cycles per 16 columns and 8 KB of weights, 64
// bytes a cycle and SM, nearly three times what HBM delivers (25 rows x 32 256 x 7168: 76 us, 92 % of the measured copy rate).
// The tensor cores truncate when they add to an accumulator: the products over 512 columns are taken out and added in ordinary
// fp32 (registers of the epilogue's threads) while the next 512 run into the other accumulator.  With one accumulator over all of
// 7168 columns the results were 2.3e-6 off a 64-bit product's, relative, and 1.2e-7 with segments.
// An accumulator lane is a row, so a thread of the epilogue sums over its tile's tokens by itself; each half tile leaves
// (m, sum 2^t, sum 2^t t), t = (z - m) log2(e), in the scratch, and a second kernel joins a row's halves.
#include "head_score.h"

#include <algorithm>

#include "pair.cuh"
#include "two.cuh"

namespace hs {

using namespace fwd;
using namespace pr;
using namespace tw;

constexpr int TM = 128, TN = 256, A_BYTES = TM * 128;
// PAIR: two blocks of a cluster work on 256 rows, each with its 128 of them and half of the tile's tokens in shared memory.
template <bool PAIR> struct Cfg {
    static constexpr int B_BYTES = (PAIR ? TN / 2 : TN) * 128, STAGE = A_BYTES + B_BYTES, STAGES = PAIR ? 6 : 4;
};
constexpr int SEG_SCORE = 8;               // k blocks of 64 columns accumulated inside the tensor cores
// Where the epilogue has twice the work (KEEP), segments twice as long give it the time: the loss's pass over 4093 rows x 151 936 x 1536 took
// 1508 us with 8 blocks, 1341 with 12 or 16, over 2048 x 32 000 x 4096 371, 356 and 341.  (Losses are then 2.2e-7 off, relative.)
constexpr int SEG_KEEP = 16;
constexpr int EPI_WARPS = 8, THREADS_H = 32 * (EPI_WARPS + 2), SMEM_H = 192 * 1024 + 1024;
static_assert(Cfg<true>::STAGE * Cfg<true>::STAGES == 192 * 1024 && Cfg<false>::STAGE * Cfg<false>::STAGES == 192 * 1024, "the stages");
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float NO_REF = -3.402823466e38f, SLACK = 11.f, FAR = -1000.f;
constexpr float OUTSIDE = -1e30f;          // a logit past the vocabulary, or below this by its bias: 2^t is 0, and t finite

// A share 2^t, t at most 0, is kept as 16 of the bits of 2^t KEEP_DOWN: 6 exponent and 10 mantissa bits (there is no sign, and no exponent above
// that of 1), so that 11 bits of it are right down to 2^-62, 43 nats below the half tile's largest.  fp16's 5 exponent bits were not enough: 14 nats
// below, dhead's row of a token that is rare in all rows was 2 % off, from 18 on it was 0.
constexpr float KEEP_DOWN = 0x1p-64f, KEEP_UP = 0x1p64f;
constexpr uint32_t KEEP_MASK = 0xffffu << 13;
struct Part { float m, S, S2, pad; };

struct KArgs {
    int32_t rows, vocab, nkb, bn, mt, nt, a_rows;
    const int32_t *tokens, *bias_ids;
    float bias;
    Part *part;                            // [rows][2 * nt]
    float *ztok;                           // [rows]
    uint16_t *keep;                        // [rows][ld_keep], or NULL: 2^t in codes (see KEEP_DOWN)
    int32_t ld_keep;
};

struct Run {                               // a thread's running sums
    float m = NO_REF, S = 0.f, S2 = 0.f;
    __device__ void raise(float to) {
        const float d = fmaxf((m - to) * LOG2E, FAR), r = ex2(d);
        S2 = r * fmaf(S, d, S2);
        S *= r;
        m = to;
    }
    __device__ void join(const Part &p) {
        const float to = fmaxf(m, p.m);
        raise(to);
        const float d = fmaxf((p.m - to) * LOG2E, FAR), r = ex2(d);
        S = fmaf(r, p.S, S);
        S2 = fmaf(r, fmaf(p.S, d, p.S2), S2);
    }
};

// Persistent: block b computes the tiles b, b + grid, ...; row tiles vary fastest, so that the blocks that run together share
// their weights in L2.  Warps 0..7 epilogues (warp w reads accumulator lanes 32 (w % 4) .., the first or second half of the
// tile's tokens), warp 8 copies, warp 9 tensor cores.
// KEEP: 2^t is kept besides, t relative to the half tile's maximum; the row's token is left out of maximum and sums (it has its logit in ztok).
template <bool PAIR, bool KEEP>
__global__ void __launch_bounds__(THREADS_H, 1) k_head_score(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                             const KArgs a) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    constexpr int STAGES = Cfg<PAIR>::STAGES, STAGE = Cfg<PAIR>::STAGE, SEG = KEEP ? SEG_KEEP : SEG_SCORE;
    __shared__ uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int32_t gave_up;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    unsigned char *smem = smem_raw + (-(int)smem_u32(smem_raw) & 1023);      // (the same in both blocks of a pair)
    const int rank = PAIR ? blockIdx.x & 1 : 0, worker = PAIR ? blockIdx.x >> 1 : blockIdx.x, workers = PAIR ? gridDim.x >> 1 : gridDim.x;
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (int i = 0; i < STAGES; ++i) { mbar_init(full + i, 1); mbar_init(empty + i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(acc_full + i, 1); mbar_init(acc_empty + i, PAIR ? 2 * EPI_WARPS : EPI_WARPS); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    if (warp == 9) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();                                          // (both blocks' barriers are set up)
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = tmem_slot;
    const int tiles = a.mt * a.nt;

    if (warp == 8) {
        // lane 0 copies hidden rows, lane 1 the head, by one instruction
        uint64_t policy;
        if (a.mt == 1 && !KEEP) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));   // (the products read it again)
        else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
        if (lane == 0) asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(policy));
        const uint32_t full0 = PAIR ? first_block(full) : smem_u32(full);
        int n = 0;
        bool ok = true;
        for (int t = worker; t < tiles && ok; t += workers) {
            const int y = lane ? (t / a.mt) * a.bn + (PAIR ? rank * (a.bn >> 1) : 0) : (t % a.mt) * (PAIR ? 2 * TM : TM) + rank * TM;
            for (int kb = 0; kb < a.nkb; ++kb, ++n) {
                const int slot = n % STAGES;
                ok = __all_sync(0xffffffffu, wait_h(&gave_up, empty + slot, (((uint32_t)(n / STAGES)) & 1u) ^ 1u));
                if (!ok) break;
                if (lane == 0 && rank == 0) mbar_expect_tx(full + slot, (uint32_t)(PAIR ? 2 * a.a_rows + a.bn : a.a_rows + a.bn) * 128u);   // (both blocks' bytes)
                if (lane < 2) tma_2d<PAIR>(smem + slot * STAGE + lane * A_BYTES, lane ? &map_b : &map_a, kb * 64, y, full0 + slot * 8, policy);
            }
        }
        // no copy may be in flight when the block ends (a pair's arrive at its first block's barriers; the second ends after it)
        for (int j = max(0, n - STAGES); j < n && rank == 0 && lane == 0; ++j)
            for (unsigned it = 0; it < MBAR_SPIN_LIMIT && !mbar_try_wait(full + j % STAGES, ((uint32_t)(j / STAGES)) & 1u); ++it) {}
    } else if (warp == 9) {
        // (all lanes wait, one issues; of a pair the first block's)
        const uint32_t on = elect_lane(), idesc = PAIR ? (umma_idesc(a.bn) & ~(31u << 24)) | (256u >> 4) << 24 : umma_idesc(a.bn);
        int n = 0, i = 0;
        bool ok = true;
        for (int t = worker; t < tiles && ok && rank == 0; t += workers, ++i) {
            for (int kb = 0; kb < a.nkb; ++kb, ++n) {
                if (kb % SEG == 0) {
                    if (kb) { PAIR ? umma2_commit_if(on, acc_full + (i & 1)) : umma_commit_if(on, acc_full + (i & 1)); ++i; }
                    ok = __all_sync(0xffffffffu, wait_h(&gave_up, acc_empty + (i & 1), (((uint32_t)(i >> 1)) & 1u) ^ 1u));
                    if (!ok) break;
                }
                const uint32_t acc = tmem + (uint32_t)(i & 1) * 256u;
                const int slot = n % STAGES;
                ok = __all_sync(0xffffffffu, wait_h(&gave_up, full + slot, ((uint32_t)(n / STAGES)) & 1u));
                if (!ok) break;
                tc_fence_after();
                const uint32_t a0 = smem_u32(smem + slot * STAGE), b0 = a0 + A_BYTES;
#pragma unroll
                for (int k16 = 0; k16 < 4; ++k16) {
                    const uint64_t da = umma_desc(a0 + k16 * 32), db = umma_desc(b0 + k16 * 32);
                    const uint32_t add = (kb % SEG > 0 || k16 > 0) ? 1u : 0u;
                    PAIR ? umma2_if(on, acc, da, db, idesc, add) : umma_if(on, acc, da, db, idesc, add);
                }
                PAIR ? umma2_commit_if(on, empty + slot) : umma_commit_if(on, empty + slot);
            }
            if (ok) PAIR ? umma2_commit_if(on, acc_full + (i & 1)) : umma_commit_if(on, acc_full + (i & 1));
        }
    } else {
        const int quad = warp & 3, half = warp >> 2;
        const int chunks = (a.bn + 31) >> 5, c0 = half ? (chunks + 1) >> 1 : 0, c1 = half ? chunks : (chunks + 1) >> 1;
        int i = 0;                                                    // segments so far
        bool ok = true;                                               // (once a wait has given up, the tiles left become NaN)
        for (int t = worker; t < tiles; t += workers) {
            const int m = t % a.mt, nti = t / a.mt, n0 = nti * a.bn, width = min(a.bn, a.vocab - n0);
            const int rq = m * (PAIR ? 2 * TM : TM) + rank * TM + quad * 32, r = rq + lane;
            const bool live = r < a.rows, reads = rq < a.rows;      // (a warp without rows has nothing to read)
            const int tok = live && a.tokens ? a.tokens[r] - n0 : -1, bid = live && a.bias_ids ? a.bias_ids[r] - n0 : -1;
            float z[4][32];                                           // this thread's logits: row r, tokens n0 + 32 (c0 + ..)
            for (int kb = 0; kb < a.nkb && ok; kb += SEG, ++i) {
                ok = __all_sync(0xffffffffu, wait_h(&gave_up, acc_full + (i & 1), ((uint32_t)(i >> 1)) & 1u));
                tc_fence_after();
                const uint32_t acc = tmem + (uint32_t)(i & 1) * 256u + ((uint32_t)(quad * 32) << 16);
                if (ok && reads)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (c0 + c < c1) {
                            uint32_t raw[32];
                            tmem_ld32(acc + (c0 + c) * 32u, raw);
#pragma unroll
                            for (int e = 0; e < 32; ++e) z[c][e] = kb ? z[c][e] + __uint_as_float(raw[e]) : __uint_as_float(raw[e]);
                        }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {                                      // the next products may overwrite the accumulator
                    if (PAIR) acc_release(acc_empty + (i & 1));
                    else mbar_arrive(acc_empty + (i & 1));
                }
            }
            Run s;
            if (ok && reads)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int at = (c0 + c) * 32, left = width - at;
                    if (c0 + c >= c1 || left <= 0) continue;
                    float (&v)[32] = z[c];
                    if ((uint32_t)(bid - at) < 32u)
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] += bid - at == e ? a.bias : 0.f;
                    if ((uint32_t)(tok - at) < 32u && tok < width) {
                        float x = 0.f;
#pragma unroll
                        for (int e = 0; e < 32; ++e) x = tok - at == e ? v[e] : x;
                        a.ztok[r] = x;
                    }
                    if ((uint32_t)(bid - at) < 32u)                   // (a bias of -infinity, say)
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = bid - at == e && v[e] < OUTSIDE ? OUTSIDE : v[e];
                    if (left < 32)                                    // columns past the vocabulary
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = e < left ? v[e] : OUTSIDE;
                    if (KEEP) {
                        if ((uint32_t)(tok - at) < 32u)
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] = tok - at == e ? OUTSIDE : v[e];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) s.m = max3(s.m, v[e], v[e + 1]);
                        continue;
                    }
                    float top = v[0];
#pragma unroll
                    for (int e = 1; e < 32; ++e) top = fmaxf(top, v[e]);
                    if (top > s.m + SLACK) s.raise(top);
                    float S0 = 0.f, S1 = 0.f, q0 = 0.f, q1 = 0.f;
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        const float t0 = (v[e] - s.m) * LOG2E, t1 = (v[e + 1] - s.m) * LOG2E, x0 = ex2(t0), x1 = ex2(t1);
                        S0 += x0; S1 += x1;
                        q0 = fmaf(x0, t0, q0); q1 = fmaf(x1, t1, q1);
                    }
                    s.S += S0 + S1;
                    s.S2 += q0 + q1;
                }
            if (KEEP && ok && reads)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int at = (c0 + c) * 32;
                    if (c0 + c >= c1 || width - at <= 0) continue;
                    Two sum = two(0.f, 0.f);
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float x0, x1;
                        apart(mul2(add2(two(z[c][e], z[c][e + 1]), two(-s.m, -s.m)), two(LOG2E, LOG2E)), x0, x1);
                        x0 = ex2(x0);
                        x1 = ex2(x1);
                        sum = add2(sum, two(x0, x1));
                        apart(mul2(two(x0, x1), two(KEEP_DOWN, KEEP_DOWN)), x0, x1);
                        w[e >> 1] = __byte_perm(__float_as_uint(x0) * 8u + 0x8000u, __float_as_uint(x1) * 8u + 0x8000u, 0x7632);
                    }
                    float S0, S1;
                    apart(sum, S0, S1);
                    s.S += S0 + S1;
                    if (live) {
                        uint16_t *p = a.keep + (size_t)r * a.ld_keep + n0 + at;
                        st32(p, w);
                        st32(p + 16, w + 8);
                    }
                }
            if (live) {
                if (!ok) s.S = s.S2 = __int_as_float(0x7fffffff);
                reinterpret_cast<float4 *>(a.part)[(size_t)r * (2 * a.nt) + nti * 2 + half] = make_float4(s.m, s.S, s.S2, 0.f);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync();                                          // (nothing of one block is in use by the other)
    if (warp == 9) {
        if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// One warp per row joins its parts.
__global__ void __launch_bounds__(128) k_head_join(const KArgs a, float *logp, float *entropy, float *lse, float *loss) {
    const int row = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (row >= a.rows) return;
    const float4 *p = reinterpret_cast<const float4 *>(a.part) + (size_t)row * (2 * a.nt);
    Run s;
    for (int i = lane; i < 2 * a.nt; i += 32) {
        const float4 v = __ldcg(p + i);
        s.join(Part{v.x, v.y, v.z, 0.f});
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Part q;
        q.m = __shfl_xor_sync(~0u, s.m, o); q.S = __shfl_xor_sync(~0u, s.S, o); q.S2 = __shfl_xor_sync(~0u, s.S2, o);
        s.join(q);
    }
    if (lane) return;
    const float l2 = log2f(s.S), l = l2 * LN2;
    if (lse) lse[row] = s.m + l;
    if (entropy) entropy[row] = (l2 - s.S2 / s.S) * LN2;
    if (logp) {
        const int t = a.tokens[row];
        const float x = t >= 0 && t < a.vocab ? (__ldcg(a.ztok + row) - s.m) - l : 0.f;
        logp[row] = x;
        if (loss) loss[row] = 0.f - x;
    }
}

// The gradient of sum_r weight_r (lse_r - z_r[token_r]) with respect to the logits, in place of what k_head_score kept: a block joins its row's
// parts and takes a piece of the row.  What was kept has 11 bits, so that rounding it to bf16 after the row's factor is known is the only
// rounding that shows (2^-11 of a gradient beside 2^-8; what is below 2^-62 of its half tile's largest, the row's token left out, loses bits
// and becomes 0).  Kept in bf16 and scaled, it was rounded twice, and the products' errors were 1.7 times those of exact gradients rounded at
// the end (1.4 with one rounding).  The token's 1 - p is the others' share, and its loss log(1 + others / its own) where it has the
// largest logit: confident rows lose nothing.  low: the remainders bf16(x - bf16(x)), or NULL.
struct DzArgs {
    int32_t segs, seg;                     // pieces of a row and their columns, a multiple of 8
    uint32_t by_bn;                        // 2^32 / bn, rounded up (exact quotients below 2^32 / bn)
    const float *weight;
    float *loss;
    __nv_bfloat16 *low;
};
constexpr int THREADS_D = 256;
template <bool LOW>
__global__ void __launch_bounds__(THREADS_D) k_head_dz(const KArgs a, const DzArgs g) {
    __shared__ Part red[THREADS_D / 32];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = blockIdx.x / g.segs, at = (blockIdx.x - row * g.segs) * g.seg, lane = threadIdx.x & 31, end = min(at + g.seg, a.vocab);
    uint4 *z = reinterpret_cast<uint4 *>(a.keep + (size_t)row * a.ld_keep), *low = LOW ? reinterpret_cast<uint4 *>(g.low + (size_t)row * a.ld_keep) : nullptr;
    constexpr int STEP = THREADS_D * 8;
    int c = at + threadIdx.x * 8;
    uint4 v[4] = {};                       // (on their way while the parts are joined)
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (c + k * STEP < end) v[k] = z[(c + k * STEP) >> 3];
    const float4 *p = reinterpret_cast<const float4 *>(a.part) + (size_t)row * (2 * a.nt);
    float m = NO_REF, S = 0.f;
    for (int i = threadIdx.x; i < 2 * a.nt; i += THREADS_D) {
        const float4 v = __ldcg(p + i);
        const float to = fmaxf(m, v.x);
        S = fmaf(S, ex2(fmaxf((m - to) * LOG2E, FAR)), v.y * ex2(fmaxf((v.x - to) * LOG2E, FAR)));
        m = to;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float qm = __shfl_xor_sync(~0u, m, o), qS = __shfl_xor_sync(~0u, S, o), to = fmaxf(m, qm);
        S = fmaf(S, ex2(fmaxf((m - to) * LOG2E, FAR)), qS * ex2(fmaxf((qm - to) * LOG2E, FAR)));
        m = to;
    }
    if (lane == 0) red[threadIdx.x >> 5] = Part{m, S, 0.f, 0.f};
    __syncthreads();
    m = red[0].m;
#pragma unroll
    for (int w = 1; w < THREADS_D / 32; ++w) m = fmaxf(m, red[w].m);
    S = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS_D / 32; ++w) S = fmaf(red[w].S, ex2(fmaxf((red[w].m - m) * LOG2E, FAR)), S);
    int tok = a.tokens[row];
    if (tok >= a.vocab) tok = -1;
    const float weight = tok >= 0 ? g.weight[row] : 0.f, zt = tok >= 0 ? __ldcg(a.ztok + row) : NO_REF, rest = m;
    m = fmaxf(m, zt);
    const float others = S * ex2(fmaxf((rest - m) * LOG2E, FAR)), mine = tok >= 0 ? ex2(fmaxf((zt - m) * LOG2E, FAR)) : 0.f;
    S = others + mine;
    const float l2 = log2f(S), of_token = -weight * (others / S);
    if (at == 0 && threadIdx.x == 0 && g.loss) g.loss[row] = tok < 0 ? 0.f : zt == m ? log1pf(others) : (m - zt) + l2 * LN2;
    const int first = (a.bn + 32) >> 6 << 5;                           // tokens of a tile's first half (whole chunks of 32)
    const auto scaled = [&](int c, uint4 v) {
        const int tile = (int)__umulhi((uint32_t)c, g.by_bn), half = c - tile * a.bn >= first;             // (c / bn)
        const float t = (p[2 * tile + half].x - m) * LOG2E - l2, f = t < FAR ? 0.f : weight * ex2(t);      // (NaN stays)
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        const Two ff = two(f, f);
        uint32_t o[4], r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float2 x = make_float2(__uint_as_float(w[e] << 13 & KEEP_MASK), __uint_as_float(w[e] >> 3 & KEEP_MASK));
            apart(mul2(mul2(two(x.x, x.y), two(KEEP_UP, KEEP_UP)), ff), x.x, x.y);
            const __nv_bfloat162 b = __floats2bfloat162_rn(x.x, x.y);
            o[e] = *reinterpret_cast<const uint32_t *>(&b);
            if (LOW) {
                const __nv_bfloat162 d = __floats2bfloat162_rn(x.x - __low2float(b), x.y - __high2float(b));
                r[e] = *reinterpret_cast<const uint32_t *>(&d);
            }
        }
        z[c >> 3] = make_uint4(o[0], o[1], o[2], o[3]);
        if (LOW) low[c >> 3] = make_uint4(r[0], r[1], r[2], r[3]);
        if ((uint32_t)(tok - c) < 8u) {                                // (the token's own, by the same thread)
            const __nv_bfloat16 b = __float2bfloat16_rn(of_token);
            reinterpret_cast<__nv_bfloat16 *>(z)[tok] = b;
            if (LOW) reinterpret_cast<__nv_bfloat16 *>(low)[tok] = __float2bfloat16_rn(of_token - __bfloat162float(b));
        }
    };
    while (c < end) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k * STEP < end) scaled(c + k * STEP, v[k]);
        c += 4 * STEP;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k * STEP < end) v[k] = z[(c + k * STEP) >> 3];
    }
}

// Tokens of a tile: the width with the least waves x (width + 16).  The 16 stands for a tile's start and end: without it many rows would
// be cut into the narrowest tiles for a fraction of a wave (2048 rows x 32 000: 32 tokens instead of 256; with 16 or 64 the same widths).
static int tile_width(int mt, int vocab, int n_sm, int step) {
    int best = TN;
    int64_t best_cost = INT64_MAX;
    for (int w = TN; w >= 32; w -= step) {
        const int64_t tiles = (int64_t)mt * ((vocab + w - 1) / w), cost = (tiles + n_sm - 1) / n_sm * (w + 16);
        if (cost < best_cost) { best_cost = cost; best = w; }
    }
    return best;
}

struct Tiles { int pair, mt, bn, nt; };
// Pairs of blocks where that leaves few rows empty: they read a third less out of L2, and the power cap leaves them a higher clock
// for it (2048 rows x 32 000 x 4096: 4.9 GB and 415 us, tensor pipe 91 % active; by single blocks 7.1 GB and 474 us).
// With 32 000 tokens x 4096: 256 rows 60 us by pairs, 68 by single blocks; 384 rows (three tiles of 128) 100 and 92; 640 (five) 145 and
// 141; 1100 (nine) 229 and 237.
// keep: tiles of whole chunks of 32.
static Tiles tiles_of(int rows, int vocab, bool keep) {
    Tiles t;
    const int m128 = (rows + TM - 1) / TM;
    t.pair = m128 % 2 == 0 || m128 >= 9;
    t.mt = t.pair ? (m128 + 1) / 2 : m128;
    t.bn = tile_width(t.mt, vocab, t.pair ? 74 : 148, t.pair || keep ? 32 : 16);      // (a pair's product takes tokens by 32)
    t.nt = (vocab + t.bn - 1) / t.bn;
    return t;
}

size_t scratch_bytes(int rows, int vocab) {
    return (size_t)rows * (2 * std::max(tiles_of(rows, vocab, false).nt, tiles_of(rows, vocab, true).nt)) * sizeof(Part) + (((size_t)rows * sizeof(float) + 255) & ~(size_t)255);
}

cudaError_t run(const Args &a, void *scratch, int n_sm, cudaStream_t st, bool *no_maps) {
    static bool attr_set[64] = {};         // the opt-in is per device
    *no_maps = false;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    EncodeFn encode;
    e = encode_fn(&encode);
    if (e != cudaSuccess) return e;
    if (!encode) { *no_maps = true; return cudaSuccess; }
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = cudaFuncSetAttribute(k_head_score<false, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_H);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_head_score<true, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_H);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_head_score<false, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_H);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_head_score<true, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_H);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    const Tiles t = tiles_of(a.rows, a.vocab, a.dz != nullptr);
    KArgs k;
    k.rows = a.rows; k.vocab = a.vocab; k.nkb = (a.d + 63) / 64; k.bn = t.bn; k.mt = t.mt; k.nt = t.nt;
    k.a_rows = std::min(TM, (a.rows + 7) & ~7);
    k.tokens = a.tokens; k.bias_ids = a.bias_ids; k.bias = a.bias;
    k.part = reinterpret_cast<Part *>(scratch);
    k.ztok = reinterpret_cast<float *>(k.part + (size_t)a.rows * (2 * t.nt));
    k.keep = reinterpret_cast<uint16_t *>(a.dz); k.ld_keep = a.ld_dz;
    CUtensorMap ma, mb;
    if (!make_map(encode, &ma, a.hidden, a.ld_hidden, a.rows, a.d, k.a_rows) || !make_map(encode, &mb, a.head, a.ld_head, a.vocab, a.d, t.pair ? t.bn / 2 : t.bn)) {
        *no_maps = true;
        return cudaSuccess;
    }
    cudaLaunchConfig_t m = {};
    m.gridDim = dim3((unsigned)std::min((int64_t)(t.pair ? n_sm / 2 : n_sm), (int64_t)t.mt * t.nt) * (t.pair ? 2 : 1));
    m.blockDim = dim3(THREADS_H);
    m.dynamicSmemBytes = SMEM_H;
    m.stream = st;
    cudaLaunchAttribute two[1];
    two[0].id = cudaLaunchAttributeClusterDimension;
    two[0].val.clusterDim.x = 2; two[0].val.clusterDim.y = two[0].val.clusterDim.z = 1;
    m.attrs = two;
    m.numAttrs = t.pair ? 1 : 0;
    e = a.dz ? t.pair ? cudaLaunchKernelEx(&m, k_head_score<true, true>, ma, mb, k) : cudaLaunchKernelEx(&m, k_head_score<false, true>, ma, mb, k)
             : t.pair ? cudaLaunchKernelEx(&m, k_head_score<true, false>, ma, mb, k) : cudaLaunchKernelEx(&m, k_head_score<false, false>, ma, mb, k);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)((a.rows + 3) / 4));
    c.blockDim = dim3(128);
    DzArgs g;
    if (a.dz) {                            // rows cut into pieces while all blocks fit the SMs at once, six on each
        g.segs = std::max(1, std::min((a.vocab + 8 * THREADS_D - 1) / (8 * THREADS_D), 6 * n_sm / a.rows));
        g.seg = ((a.vocab + g.segs - 1) / g.segs + 7) & ~7;
        g.by_bn = (uint32_t)((((uint64_t)1 << 32) + t.bn - 1) / t.bn);
        g.weight = a.weight; g.loss = a.loss; g.low = reinterpret_cast<__nv_bfloat16 *>(a.dz_low);
        c.gridDim = dim3((unsigned)a.rows * (unsigned)g.segs);
        c.blockDim = dim3(THREADS_D);
    }
    c.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // it waits for the products by itself
    at[0].val.programmaticStreamSerializationAllowed = 1;
    c.attrs = at;
    c.numAttrs = 1;
    if (a.dz) return g.low ? cudaLaunchKernelEx(&c, k_head_dz<true>, k, g) : cudaLaunchKernelEx(&c, k_head_dz<false>, k, g);
    return cudaLaunchKernelEx(&c, k_head_join, k, a.logp, a.entropy, a.lse, a.loss);
}

}  // namespace hs

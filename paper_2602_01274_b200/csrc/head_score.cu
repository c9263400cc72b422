// LM head fused with the scoring of given tokens: z = hidden head^T, and of each row of z only its log-sum-exp, its entropy and
// the logit of one token.  The logits are never written: [rows][vocab] f32 would be 262 MB for 2048 rows of 32 000.
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

#include <cuda.h>

#include <algorithm>

#include "forward.cuh"

namespace hs {

using namespace fwd;

constexpr int TM = 128, TN = 256, A_BYTES = TM * 128;
// PAIR: two blocks of a cluster work on 256 rows, each with its 128 of them and half of the tile's tokens in shared memory.
template <bool PAIR> struct Cfg {
    static constexpr int B_BYTES = (PAIR ? TN / 2 : TN) * 128, STAGE = A_BYTES + B_BYTES, STAGES = PAIR ? 6 : 4;
};
constexpr int SEG = 8;                     // k blocks of 64 columns accumulated inside the tensor cores
constexpr int EPI_WARPS = 8, THREADS_H = 32 * (EPI_WARPS + 2), SMEM_H = 192 * 1024 + 1024;
static_assert(Cfg<true>::STAGE * Cfg<true>::STAGES == 192 * 1024 && Cfg<false>::STAGE * Cfg<false>::STAGES == 192 * 1024, "the stages");
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float NO_REF = -3.402823466e38f, SLACK = 11.f, FAR = -1000.f;
constexpr float OUTSIDE = -1e30f;          // a logit past the vocabulary: 2^t is 0, and t finite

struct Part { float m, S, S2, pad; };

struct KArgs {
    int32_t rows, vocab, nkb, bn, mt, nt, a_rows;
    const int32_t *tokens, *bias_ids;
    float bias;
    Part *part;                            // [rows][2 * nt]
    float *ztok;                           // [rows]
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// bar: a shared::cluster address; with PAIR that of the pair's first block.
template <bool PAIR>
__device__ __forceinline__ void tma_2d(void *dst, const CUtensorMap *map, int x, int y, uint32_t bar, uint64_t policy) {
    if (PAIR)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;"
                     ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(bar), "l"(policy) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;"
                     ::"r"(smem_u32(dst)), "l"(map), "r"(x), "r"(y), "r"(bar), "l"(policy) : "memory");
}
__device__ __forceinline__ uint32_t first_block(const void *smem) {      // the address of the pair's first block
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(smem)), "r"(0));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// As umma_if and umma_commit_if for both blocks' operands, accumulators and barriers; issued by the first block.
__device__ __forceinline__ void umma2_if(uint32_t on, uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
                 "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}\n"
                 ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(on) : "memory");
}
__device__ __forceinline__ void umma2_commit_if(uint32_t on, uint64_t *bar) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
                 "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %2;\n\t}"
                 ::"r"(smem_u32(bar)), "r"(on), "h"((uint16_t)3) : "memory");
}
// Bounded wait; one that runs out ends the block's work (its rows become NaN).
__device__ __forceinline__ bool wait_h(volatile int32_t *gave_up, uint64_t *bar, uint32_t parity) {
    for (unsigned it = 1; !mbar_try_wait(bar, parity); ++it)
        if ((it & 1023u) == 0 && (it > MBAR_SPIN_LIMIT || *gave_up)) { *gave_up = 1; return false; }
    return true;
}

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
template <bool PAIR>
__global__ void __launch_bounds__(THREADS_H, 1) k_head_score(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                             const KArgs a) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    constexpr int STAGES = Cfg<PAIR>::STAGES, STAGE = Cfg<PAIR>::STAGE;
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
        if (lane == 0) {
            uint64_t keep, stream;
            asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(keep));
            if (a.mt == 1) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(stream));
            else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(stream));
            int n = 0;
            bool ok = true;
            for (int t = worker; t < tiles && ok; t += workers) {
                const int r0 = (t % a.mt) * (PAIR ? 2 * TM : TM) + rank * TM, n0 = (t / a.mt) * a.bn + (PAIR ? rank * (a.bn >> 1) : 0);
                for (int kb = 0; kb < a.nkb; ++kb, ++n) {
                    const int slot = n % STAGES;
                    ok = wait_h(&gave_up, empty + slot, (((uint32_t)(n / STAGES)) & 1u) ^ 1u);
                    if (!ok) break;
                    unsigned char *st = smem + slot * STAGE;
                    if (rank == 0) mbar_expect_tx(full + slot, (uint32_t)(PAIR ? 2 * a.a_rows + a.bn : a.a_rows + a.bn) * 128u);   // (both blocks' bytes)
                    const uint32_t bar = PAIR ? first_block(full + slot) : smem_u32(full + slot);
                    tma_2d<PAIR>(st, &map_a, kb * 64, r0, bar, keep);
                    tma_2d<PAIR>(st + A_BYTES, &map_b, kb * 64, n0, bar, stream);
                }
            }
            // no copy may be in flight when the block ends (a pair's arrive at its first block's barriers; the second ends after it)
            for (int j = max(0, n - STAGES); j < n && rank == 0; ++j)
                for (unsigned it = 0; it < MBAR_SPIN_LIMIT && !mbar_try_wait(full + j % STAGES, ((uint32_t)(j / STAGES)) & 1u); ++it) {}
        }
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
                    if (PAIR) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(first_block(acc_empty + (i & 1))) : "memory");
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
                    if (left < 32)                                    // columns past the vocabulary
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = e < left ? v[e] : OUTSIDE;
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
__global__ void __launch_bounds__(128) k_head_join(const KArgs a, float *logp, float *entropy, float *lse) {
    const int row = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
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
        logp[row] = t >= 0 && t < a.vocab ? (__ldcg(a.ztok + row) - s.m) - l : 0.f;
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
static Tiles tiles_of(int rows, int vocab) {
    Tiles t;
    const int m128 = (rows + TM - 1) / TM;
    t.pair = m128 % 2 == 0 || m128 >= 9;
    t.mt = t.pair ? (m128 + 1) / 2 : m128;
    t.bn = tile_width(t.mt, vocab, t.pair ? 74 : 148, t.pair ? 32 : 16);      // (a pair's product takes tokens by 32)
    t.nt = (vocab + t.bn - 1) / t.bn;
    return t;
}

size_t scratch_bytes(int rows, int vocab) {
    return (size_t)rows * (2 * tiles_of(rows, vocab).nt) * sizeof(Part) + (((size_t)rows * sizeof(float) + 255) & ~(size_t)255);
}

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                             const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// bf16 [rows][d], boxes of `box` rows x 64 columns in the 128-byte swizzle; what lies outside reads as 0.
static bool make_map(EncodeFn encode, CUtensorMap *map, const void *p, int64_t ld, int rows, int d, int box) {
    const cuuint64_t dims[2] = {(cuuint64_t)d, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t boxes[2] = {64, (cuuint32_t)box}, one[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(p), dims, strides, boxes, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t run(const Args &a, void *scratch, int n_sm, cudaStream_t st, bool *no_maps) {
    static bool attr_set[64] = {};         // the opt-in is per device
    static EncodeFn encode = nullptr;
    *no_maps = false;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!encode) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult q;
        e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
        if (e != cudaSuccess) return e;
        if (q != cudaDriverEntryPointSuccess || !fn) { *no_maps = true; return cudaSuccess; }
        encode = reinterpret_cast<EncodeFn>(fn);
    }
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = cudaFuncSetAttribute(k_head_score<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_H);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(k_head_score<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_H);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    const Tiles t = tiles_of(a.rows, a.vocab);
    KArgs k;
    k.rows = a.rows; k.vocab = a.vocab; k.nkb = (a.d + 63) / 64; k.bn = t.bn; k.mt = t.mt; k.nt = t.nt;
    k.a_rows = std::min(TM, (a.rows + 7) & ~7);
    k.tokens = a.tokens; k.bias_ids = a.bias_ids; k.bias = a.bias;
    k.part = reinterpret_cast<Part *>(scratch);
    k.ztok = reinterpret_cast<float *>(k.part + (size_t)a.rows * (2 * t.nt));
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
    e = t.pair ? cudaLaunchKernelEx(&m, k_head_score<true>, ma, mb, k) : cudaLaunchKernelEx(&m, k_head_score<false>, ma, mb, k);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)((a.rows + 3) / 4));
    c.blockDim = dim3(128);
    c.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // it waits for the products by itself
    at[0].val.programmaticStreamSerializationAllowed = 1;
    c.attrs = at;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, k_head_join, k, a.logp, a.entropy, a.lse);
}

}  // namespace hs

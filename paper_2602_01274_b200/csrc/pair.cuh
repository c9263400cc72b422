// Pairs of blocks on the tensor cores: what the kernels on an LM head share.
#pragma once
#include <cuda.h>

#include "forward.cuh"

namespace pr {

using namespace fwd;

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
// A warp's accumulator values are in registers (tcgen05.wait::ld): the next products may overwrite them.  Called by one lane for the first block's
// barrier.  Relaxed: nothing else is handed over, and an arrival that releases at cluster scope waits for the warp's stores to global memory
// (both gradients' products for 33 rows x 32 000 x 768: 28.8 us, 27.1 relaxed).
__device__ __forceinline__ void acc_release(uint64_t *bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(first_block(bar)) : "memory");
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
__device__ __forceinline__ void st32(void *p, const uint32_t *v) {         // 32 bytes, aligned
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]),
                 "r"(v[6]), "r"(v[7]) : "memory");
}
// Bounded wait; one that runs out ends the block's work (its rows become NaN).
__device__ __forceinline__ bool wait_h(volatile int32_t *gave_up, uint64_t *bar, uint32_t parity, unsigned limit = MBAR_SPIN_LIMIT) {
    for (unsigned it = 1; !mbar_try_wait(bar, parity); ++it)
        if ((it & 1023u) == 0 && (it > limit || *gave_up)) { *gave_up = 1; return false; }
    return true;
}

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                             const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// *encode: nullptr where the driver has none.
static cudaError_t encode_fn(EncodeFn *encode) {
    static EncodeFn found = nullptr;
    *encode = found;
    if (found) return cudaSuccess;
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
    if (e != cudaSuccess) return e;
    if (q == cudaDriverEntryPointSuccess && fn) *encode = found = reinterpret_cast<EncodeFn>(fn);
    return cudaSuccess;
}

// bf16 [rows][d], boxes of `box` rows x 64 columns in the 128-byte swizzle; what lies outside reads as 0 and is not written.
static bool make_map(EncodeFn encode, CUtensorMap *map, const void *p, int64_t ld, int64_t rows, int d, int box) {
    const cuuint64_t dims[2] = {(cuuint64_t)d, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t boxes[2] = {64, (cuuint32_t)box}, one[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(p), dims, strides, boxes, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace pr

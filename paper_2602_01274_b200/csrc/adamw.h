// AdamW over many tensors at once: host interface (kernels: adamw.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/pacer.h"

namespace ow {

constexpr int NORM_BLOCKS = 1184;          // blocks of the norm's kernel at most: eight an SM
constexpr int NORM_CAP = 1024;             // tensors a launch

size_t norm_scratch_bytes(int n);
cudaError_t grad_norm(const pacer_gradient *tbl, int n, float *norm, double *scratch, cudaStream_t st);
cudaError_t adamw(const pacer_adamw_tensor *tbl, int n, const pacer_adamw_cfg &cfg, cudaStream_t st);
cudaError_t states(const pacer_adamw_tensor *tbl, int n, float *const *exp_avg, float *const *exp_avg_sq, cudaStream_t st);

}  // namespace ow

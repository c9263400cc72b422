// Gradients of the LM head fused with the scoring: host interface (kernels: head_grad.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "head_score.h"

namespace hg {

struct Args {
    const void *hidden, *head;             // bf16 [rows][d], [vocab][d]
    int64_t ld_hidden, ld_head;
    int32_t rows, vocab, d;
    const int32_t *tokens, *bias_ids;      // [rows], each may be NULL
    float bias;
    const float *logp, *lse, *entropy;     // [rows]; entropy only with g_entropy
    const float *g_logp, *g_entropy, *g_lse;   // [rows], each may be NULL
    float sign;                            // of g_logp
    void *dhidden, *dhead;                 // bf16, each may be NULL
    int64_t ld_dhidden, ld_dhead;
};

size_t scratch_bytes(int rows, int vocab, int d, int n_sm);
// Sets *no_maps where the driver cannot describe the operands to the copy engine.  after: the kernels before it in the stream are this library's own
// and let their successor be set up early.
cudaError_t run(const Args &a, void *scratch, int n_sm, bool after, cudaStream_t st, bool *no_maps);

// Loss (may be NULL) and, with g_logp = -1 times a weight, the gradients in one call; logp and lse of `a` are not read.
size_t nll_scratch_bytes(int rows, int vocab, int d, int n_sm);
cudaError_t run_nll(const Args &a, float *loss, void *scratch, int n_sm, cudaStream_t st, bool *no_maps);

}  // namespace hg

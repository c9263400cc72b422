// LM head fused with the scoring of given tokens: host interface (kernels: head_score.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace hs {

constexpr int MAX_ROWS = 1 << 20, MAX_VOCAB = 1 << 21, MAX_D = 1 << 16;

struct Args {
    const void *hidden, *head;             // bf16 [rows][d], [vocab][d]
    int64_t ld_hidden, ld_head;
    int32_t rows, vocab, d;
    const int32_t *tokens, *bias_ids;      // [rows]; bias_ids may be NULL
    float bias;
    float *logp, *entropy, *lse;           // [rows], each may be NULL
};

size_t scratch_bytes(int rows, int vocab);
// Sets *no_maps where the driver cannot describe the operands to the copy engine.
cudaError_t run(const Args &a, void *scratch, int n_sm, cudaStream_t st, bool *no_maps);

}  // namespace hs

// Operators on rows of logits: host interface (kernels: logits.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace lg {

constexpr int MAX_TOP = 128;               // alternatives of a row at most
constexpr int MAX_VOCAB = 3 << 17, MAX_ROWS = 1 << 24;
constexpr int MAX_K = 256;                 // entries of a teacher's list at most

struct Rows {                              // [rows][vocab] with `ld` elements from row to row
    const void *z;
    int32_t dtype;                         // PACER_F32 / _BF16 / _F16
    int64_t ld;
    int32_t rows, vocab;
};

// Rows of a verify window, in place of tokens[row]: row = seq * per_seq + j is left alone from n_rows[seq] on; before that its
// token is drafts[seq][j], the last row (j = n_rows[seq] - 1) has none.
struct Window {
    const int32_t *n_rows;                 // NULL: ordinary call
    const int32_t *drafts;                 // [seq][per_seq - 1]
    int32_t per_seq;
};

struct ScoreOut {                          // each may be NULL; [rows], top_*: [rows][top]
    float *logp, *entropy, *lse;
    int32_t top;
    int32_t *top_ids;
    float *top_logp;
};

cudaError_t logprobs(const Rows &r, const int32_t *tokens, const Window &win, const ScoreOut &out, cudaStream_t st);

cudaError_t logprobs_backward(const Rows &r, const int32_t *tokens, const float *lse, const float *entropy, const float *g_logp,
                              const float *g_entropy, const float *g_lse, void *dz, int64_t ld_dz, cudaStream_t st);

struct Teacher {
    const int32_t *ids;                    // [rows][k], an entry outside [0, vocab) is none
    const void *t;                         // [rows][k]
    int32_t dtype, k;
    const float *lse;                      // [rows] or NULL: the list is renormalised
    float temp, inv_temp;                  // the temperature and one over it
};

// loss, lse, tail_lse: [rows], each may be NULL.  dz (may be NULL): weight[row] times the gradient of loss[row].
cudaError_t distill(const Rows &r, const Teacher &t, float *loss, float *lse, float *tail_lse, const float *weight, void *dz, int64_t ld_dz,
                    cudaStream_t st);
cudaError_t distill_backward(const Rows &r, const Teacher &t, const float *lse, const float *tail_lse, const float *weight, void *dz,
                             int64_t ld_dz, cudaStream_t st);

}  // namespace lg

// Internal declarations of the operators that teach a probe: row norms and their
// backward pass, and the cross entropy over a vocabulary with its gradients.
#pragma once

#include "sp_cache.cuh"

namespace sp {

// ---------------------------------------------------------------------------
struct NormArgs {
    int n, d, dtype, out_dtype;
    float eps;
    long long xs, rs, ss, ys;      // elements from a row to the next
    const void *x, *r;             // r: added to x, or NULL
    const float *gain;             // or NULL
    void *sum, *y;                 // sum: or NULL
    float *y_scale;                // of 8-bit rows
};
struct NormBackArgs {
    int n, d, dtype;
    float eps;
    long long xs, rs, ss, ys;      // of grad_x, grad_sum, sum, grad_y
    const void *dy, *s, *ds;       // ds: or NULL
    const float *gain;             // or NULL
    void *dx;
    float *dgain;                  // or NULL
    float *part;                   // [norm_back_parts][d], for dgain
};
cudaError_t launch_norm(const NormArgs &a, cudaStream_t st);
// Partial rows of the gain's gradient.
int norm_back_parts(int n, int d, int n_sm);
cudaError_t launch_norm_backward(const NormBackArgs &a, int n_sm, cudaStream_t st);

// ---------------------------------------------------------------------------
// Tokens that have a target are counted off first: row `pos` of the products is token keep[pos].
struct VocabRow {
    float lse2, g;                 // log sum in log2 units and the loss's gradient (backward)
    int target, token;
};
struct VocabArgs {
    int n, V, d, dtype;
    long long hs, ws;              // elements from a row of h and of w (of their gradients) to the next
    const void *h, *w;
    const int *targets;
    // forward
    float *loss, *lse;
    // backward
    const float *lse_in, *dloss;   // dloss: or NULL = ones
    void *dh, *dw;                 // dw: or NULL
    // workspace
    int *count;                    // tokens kept
    VocabRow *rows;                // [n]
    bf16 *hc;                      // tensor cores: [pad][d] kept tokens' rows, then zeros
    int pad;                       // n rounded up to whole tiles
    float2 *part;                  // forward: [n][parts] (max in log2 units, sum) of a piece of the vocabulary
    float *at;                     // forward: [n] the target's logit, log2 units
    int parts;
    void *grad;                    // backward: [pad][piece] of dloss (p - 1_t), bf16 or float
    int piece, n_pieces;           // vocabulary rows of a piece
    float *acc;                    // backward: [planes][n][d] of dh
    int planes;
    int *status;
};
// CUDA cores: fp32 arithmetic, any alignment.
void plan_vocab_simt(VocabArgs *a, bool backward);
cudaError_t launch_vocab_loss_simt(const VocabArgs &a, cudaStream_t st);
cudaError_t launch_vocab_backward_simt(const VocabArgs &a, cudaStream_t st);
// tcgen05: bf16, rows of h and w in whole 16-byte vectors.
bool vocab_tc_supported(const VocabArgs &a);
void plan_vocab_tc(VocabArgs *a, bool backward, int n_sm);
cudaError_t launch_vocab_loss_tc(const VocabArgs &a, int n_sm, cudaStream_t st);
cudaError_t launch_vocab_backward_tc(const VocabArgs &a, int n_sm, cudaStream_t st);
// The steps around the products, shared by both.
cudaError_t launch_vocab_keep(const VocabArgs &a, bool backward, cudaStream_t st);
cudaError_t launch_vocab_finish_loss(const VocabArgs &a, cudaStream_t st);
cudaError_t launch_vocab_finish_dh(const VocabArgs &a, cudaStream_t st);

}  // namespace sp

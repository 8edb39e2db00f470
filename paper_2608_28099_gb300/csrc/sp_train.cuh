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
cudaError_t launch_norm(const NormArgs &a, int n_sm, cudaStream_t st);
// Partial rows of the gain's gradient.
int norm_back_parts(int n, int d, int n_sm);
cudaError_t launch_norm_backward(const NormBackArgs &a, int n_sm, cudaStream_t st);

// ---------------------------------------------------------------------------
// Tokens that have a target are counted off first: row `pos` of the products is token keep[pos].
struct VocabRow {
    float lse, g;                  // log sum and the loss's gradient (backward)
    int target, token;
};
// dh's tiles for the tokens kept, and their splits along the vocabulary (none is empty).
struct DhPlan {
    int kept, m_tiles, splits, per;  // per: k-blocks of a split
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
    DhPlan *count;                 // tokens kept, and how dh is cut for them (backward)
    VocabRow *rows;                // [n]
    void *hc;                      // [pad][d] kept tokens' rows (tensor cores: then zeros)
    int tensor;                    // which kernels
    int tm;                        // rows of a tile of dh (CUDA cores: rows and columns of any)
    int pad;                       // n rounded up to whole tiles
    int tn;                        // forward, tensor cores: vocabulary rows of a tile
    int box;                       // tensor cores: rows of the tokens that a CTA copies a k-block (up to 128 tokens fewer)
    int direct;                    // forward, tensor cores, one tile of tokens: they are not counted off, row m
                                   // of the products is token m
    float2 *part;                  // forward: [n][parts] (max, sum of exponentials) of a piece of the vocabulary
    float *at;                     // forward: [n] the target's logit
    int parts;
    void *grad;                    // backward: [pad][piece] of dloss (p - 1_t), bf16 or float
    int piece, n_pieces;           // vocabulary rows of a piece
    float *acc;                    // backward: [splits][rows][d] of dh, rows: whole tiles of kept tokens
    long long acc_rows;            // splits x rows, at most
    int pairs;                     // pairs of CTAs (tensor cores), or blocks, that dh's splits are balanced over
    int *status;
};
__host__ __device__ inline bool has_target(int t, int V) { return t >= 0 && t < V; }
// CUDA cores: fp32 arithmetic, any alignment.
void plan_vocab_simt(VocabArgs *a, bool backward, int n_sm);
cudaError_t launch_vocab_loss_simt(const VocabArgs &a, cudaStream_t st);
cudaError_t launch_vocab_backward_simt(const VocabArgs &a, cudaStream_t st);
// tcgen05: bf16, rows of h and w in whole 16-byte vectors.
bool vocab_tc_supported(const VocabArgs &a);
void plan_vocab_tc(VocabArgs *a, bool backward, int n_sm);
cudaError_t launch_vocab_loss_tc(const VocabArgs &a, cudaStream_t st);
cudaError_t launch_vocab_backward_tc(const VocabArgs &a, cudaStream_t st);
// The steps around the products, shared by both.
cudaError_t launch_vocab_keep(const VocabArgs &a, bool backward, cudaStream_t st);
cudaError_t launch_vocab_finish_loss(const VocabArgs &a, cudaStream_t st);
cudaError_t launch_vocab_finish_dh(const VocabArgs &a, cudaStream_t st);

}  // namespace sp

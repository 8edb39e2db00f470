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
    void *hc;                      // [pad][d] kept tokens' rows (tensor cores: then zeros)
    int tensor;                    // which kernels
    int pad;                       // n rounded up to whole tiles
    int tn;                        // forward, tensor cores: vocabulary rows of a tile
    int direct;                    // forward, tensor cores, one tile of tokens: they are not counted off, row m
                                   // of the products is token m
    float2 *part;                  // forward: [n][parts] (max, sum of exponentials) of a piece of the vocabulary
    float *at;                     // forward: [n] the target's logit
    int parts;
    void *grad;                    // backward: [pad][piece] of dloss (p - 1_t), bf16 or float
    int piece, n_pieces;           // vocabulary rows of a piece
    float *acc;                    // backward: [splits][rows][d] of dh, rows: whole tiles of kept tokens
    long long acc_rows;            // splits x rows, at most
    int pairs;                     // pairs of CTAs (tensor cores), or SMs, that split_count balances over
    int *status;
};
__host__ __device__ inline bool has_target(int t, int V) { return t >= 0 && t < V; }
// Splits along the vocabulary of dh's tiles (tm rows a tile) over `units` of the machine, the same on the
// host (for all counts) and on the device (for the one it is): the fewest rounds of k-blocks, a split's
// partial costing some itself (two passes over it: `plane` k-blocks a tile).
struct Splits {
    int s, per;                    // splits, k-blocks of each (none is empty)
};
__host__ __device__ inline Splits split_count(int m_tiles, int n_tiles, int kb, int units, float plane) {
    Splits best{1, kb};
    float least = 3e38f;
    if ((long long)m_tiles * n_tiles >= 8ll * units) return best;
    const int tiles = m_tiles * n_tiles;
    for (int s = 1; s <= 16; ++s) {
        const int per = ceil_div(kb, s);
        if (tiles * (s - 1) >= 8 * units || (s - 1) * per >= kb) continue;
        const float cost = (float)ceil_div(tiles * s, units) * (float)(per + 4) + plane * (float)(s - 1) * (float)tiles / (float)units;
        if (cost < least) least = cost, best = Splits{s, per};
    }
    return best;
}
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
// dh's tiles and their splits for `count` kept tokens, by either kind of kernel.
struct DhPlan {
    int m_tiles, rows;
    Splits k;
};
__host__ __device__ inline DhPlan dh_plan(const VocabArgs &a, int count) {
    const int tm = a.tensor ? 256 : 64, tn = tm, bk = a.tensor ? 64 : 32, piece = a.piece < a.V ? a.piece : a.V;
    DhPlan p;
    p.m_tiles = ceil_div(count < 1 ? 1 : count, tm);
    p.rows = p.m_tiles * tm;
    // (a k-block of 256 x 256 x 64 takes a pair 0.27 us, in which two passes over 0.3 tiles of fp32 partials fit
    // the HBM's share of a pair; of 64 x 64 x 32 some 0.7 us, which a partial does not weigh against)
    p.k = split_count(p.m_tiles, ceil_div(a.d, tn), ceil_div(piece, bk), a.pairs, a.tensor ? 24.f : 2.f);
    return p;
}

}  // namespace sp

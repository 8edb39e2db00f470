// C entry points of the row norms and of the vocabulary loss: argument checks and launches.
#include <math.h>
#include <string.h>

#include "sp_host.cuh"
#include "sp_train.cuh"

using namespace sp;

namespace {

size_t elem_bytes(int dtype) { return dtype == SP_F32 ? 4 : dtype == SP_BF16 ? 2 : 1; }

bool aligned(const void *p, size_t to) { return !((uintptr_t)p & (to - 1)); }

// Shapes of the norm; out8: 8-bit rows are a choice.
sp_status check_norm(const sp_norm_dims *d, bool out8, long long (&strides)[4]) {
    if (!d) return fail(SP_ERR_INVALID_ARG, "dims is NULL");
    if (d->n_rows < 0) return fail(SP_ERR_INVALID_ARG, "n_rows must be >= 0");
    if (d->d < 1) return fail(SP_ERR_INVALID_ARG, "d must be >= 1");
    if (d->d > 1 << 24) return fail(SP_ERR_UNSUPPORTED, "d above 2^24");
    if (!float_type(d->dtype)) return fail(SP_ERR_INVALID_ARG, "bad dtype %d", d->dtype);
    if (out8 && d->out_dtype != d->dtype && d->out_dtype != SP_E4M3)
        return fail(SP_ERR_INVALID_ARG, "out_dtype must be dtype or SP_E4M3");
    if (!(d->eps >= 0.f) || !isfinite(d->eps)) return fail(SP_ERR_INVALID_ARG, "eps must be finite and >= 0");
    const long long given[4] = {d->x_stride, d->r_stride, d->s_stride, d->y_stride};
    for (int i = 0; i < 4; ++i) {
        strides[i] = given[i] ? given[i] : d->d;
        if (strides[i] < d->d) return fail(SP_ERR_INVALID_ARG, "a row does not fit its stride");
    }
    return SP_OK;
}

sp_status check_vocab(const sp_vocab_dims *d, bool backward, VocabArgs *a) {
    memset(a, 0, sizeof *a);
    if (!d) return fail(SP_ERR_INVALID_ARG, "dims is NULL");
    if (d->n_tokens < 0) return fail(SP_ERR_INVALID_ARG, "n_tokens must be >= 0");
    if (d->vocab < 1 || d->d_model < 1) return fail(SP_ERR_INVALID_ARG, "vocab and d_model must be >= 1");
    // (tiles are 32-bit numbers in the kernels, and one index of a grid on CUDA cores)
    if (d->n_tokens > 4000000 || d->vocab > 1 << 24 || d->d_model > 1 << 20)
        return fail(SP_ERR_UNSUPPORTED, "n_tokens above 4000000, vocab above 2^24 or d_model above 2^20");
    if (!float_type(d->dtype)) return fail(SP_ERR_INVALID_ARG, "bad dtype %d", d->dtype);
    if (d->path < 0 || d->path > 2) return fail(SP_ERR_INVALID_ARG, "bad path %d", d->path);
    a->n = d->n_tokens;
    a->V = d->vocab;
    a->d = d->d_model;
    a->dtype = d->dtype;
    a->hs = d->h_stride ? d->h_stride : d->d_model;
    a->ws = d->w_stride ? d->w_stride : d->d_model;
    if (a->hs < a->d || a->ws < a->d) return fail(SP_ERR_INVALID_ARG, "a row does not fit its stride");
    const bool tensor = d->path != 1 && vocab_tc_supported(*a);
    if (d->path == 2 && !tensor)
        return fail(SP_ERR_UNSUPPORTED, "the tensor-core kernels need bf16 and d_model, h_stride and w_stride in multiples of 8");
    if (a->n == 0) return SP_OK;
    if (tensor) plan_vocab_tc(a, backward, sm_count());
    else plan_vocab_simt(a, backward, sm_count());
    a->tensor = tensor;
    if (backward) {
        // most rows of partial dh for any number of kept tokens (see plan_dh)
        const long long tm = a->tm, m_tiles = ceil_div_ll(a->n, tm);
        const long long more = ceil_div_ll(8ll * a->pairs, ceil_div_ll(a->d, tm));
        a->acc_rows = (m_tiles + (more < 15 * m_tiles ? more : 15 * m_tiles)) * tm;
    }
    return SP_OK;
}

// Places the workspace's parts from `base` on; returns their bytes (never 0: that answers an error).
size_t lay_out(VocabArgs *a, bool backward, char *base) {
    size_t at = 0;
    const size_t es = elem_bytes(a->dtype);
    const auto take = [&](size_t bytes) {
        char *p = base + at;
        at += align256(bytes);
        return p;
    };
    a->count = (DhPlan *)take(sizeof(DhPlan));
    a->rows = (VocabRow *)take((size_t)a->n * sizeof(VocabRow));
    a->hc = take((size_t)a->pad * a->d * es);
    if (!backward) {
        a->part = (float2 *)take((size_t)a->n * a->parts * sizeof(float2));
        a->at = (float *)take((size_t)a->n * sizeof(float));
    } else {
        a->grad = take((size_t)a->pad * a->piece * (a->tensor ? sizeof(bf16) : sizeof(float)));
        a->acc = (float *)take((size_t)a->acc_rows * a->d * sizeof(float));
    }
    return at;
}

sp_status check_vocab_buffers(VocabArgs *a, bool backward, const void *d_h, const void *d_w, const int *d_targets,
                              const void *d_dh, const void *d_dw, const float *d_lse, const float *d_loss, void *d_workspace,
                              size_t workspace_bytes) {
    if (!d_h || !d_w || !d_targets || !d_workspace) return fail(SP_ERR_INVALID_ARG, "a required pointer is NULL");
    const size_t to = a->tensor ? 16 : elem_bytes(a->dtype);
    if (!aligned(d_h, to) || !aligned(d_w, to) || !aligned(d_dh, to) || !aligned(d_dw, to))
        return fail(SP_ERR_INVALID_ARG, a->tensor ? "h, w and their gradients must be 16-byte aligned (path 1: to their type)"
                                              : "h, w and their gradients must be aligned to their type");
    if (!aligned(d_targets, 4) || !aligned(d_lse, 4) || !aligned(d_loss, 4))
        return fail(SP_ERR_INVALID_ARG, "targets, losses and log sums must be aligned to their type");
    if (!aligned(d_workspace, 256)) return fail(SP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const size_t need = lay_out(a, backward, (char *)d_workspace);
    if (workspace_bytes < need) return fail(SP_ERR_INVALID_ARG, "workspace too small (%zu < %zu)", workspace_bytes, need);
    a->h = d_h;
    a->w = d_w;
    a->targets = d_targets;
    return SP_OK;
}

}  // namespace

extern "C" {

sp_status sp_norm(sp_stream stream, const sp_norm_dims *dims, const void *d_x, const void *d_residual, const float *d_gain,
                  void *d_sum, void *d_y, float *d_y_scale) {
    long long st[4];
    sp_status s = check_norm(dims, true, st);
    if (s != SP_OK) return s;
    if (dims->n_rows == 0) return SP_OK;
    const bool out8 = dims->out_dtype == SP_E4M3;
    if (!d_x || !d_y || (out8 && !d_y_scale)) return fail(SP_ERR_INVALID_ARG, "a required pointer is NULL");
    const size_t es = elem_bytes(dims->dtype);
    if (!aligned(d_x, es) || !aligned(d_residual, es) || !aligned(d_sum, es) || !aligned(d_y, elem_bytes(dims->out_dtype)) ||
        !aligned(d_gain, 4) || !aligned(d_y_scale, 4))
        return fail(SP_ERR_INVALID_ARG, "rows, gain and scales must be aligned to their type");
    // in place: the same rows
    const bool sum_x = d_sum && d_sum == d_x, sum_r = d_sum && d_sum == d_residual, y_x = d_y == d_x, y_r = d_y == d_residual;
    if (d_y == d_sum || (out8 && (y_x || y_r)) || (sum_x && st[2] != st[0]) || (sum_r && st[2] != st[1]) ||
        (y_x && st[3] != st[0]) || (y_r && st[3] != st[1]))
        return fail(SP_ERR_INVALID_ARG, "outputs overlap each other or, in another stride or type, their inputs");
    NormArgs a{dims->n_rows, dims->d, dims->dtype, dims->out_dtype, dims->eps, st[0], st[1], st[2], st[3], d_x, d_residual,
               d_gain, d_sum, d_y, d_y_scale};
    return launched(launch_norm(a, sm_count(), (cudaStream_t)stream), "sp_norm");
}

size_t sp_norm_backward_workspace_bytes(const sp_norm_dims *dims) {
    long long st[4];
    if (check_norm(dims, false, st) != SP_OK) return 0;
    return align256((size_t)norm_back_parts(dims->n_rows > 0 ? dims->n_rows : 1, dims->d, sm_count()) * dims->d * sizeof(float));
}

sp_status sp_norm_backward(sp_stream stream, const sp_norm_dims *dims, const void *d_grad_y, const void *d_sum,
                           const float *d_gain, const void *d_grad_sum, void *d_grad_x, float *d_grad_gain, void *d_workspace,
                           size_t workspace_bytes) {
    long long st[4];
    sp_status s = check_norm(dims, false, st);
    if (s != SP_OK) return s;
    if (dims->n_rows == 0 && !d_grad_gain) return SP_OK;
    if (dims->n_rows > 0 && (!d_grad_y || !d_sum || !d_grad_x)) return fail(SP_ERR_INVALID_ARG, "a required pointer is NULL");
    const size_t es = elem_bytes(dims->dtype);
    if (!aligned(d_grad_y, es) || !aligned(d_sum, es) || !aligned(d_grad_sum, es) || !aligned(d_grad_x, es) ||
        !aligned(d_gain, 4) || !aligned(d_grad_gain, 4))
        return fail(SP_ERR_INVALID_ARG, "rows and gain must be aligned to their type");
    if ((d_grad_x == d_grad_y && st[0] != st[3]) || (d_grad_x == d_sum && st[0] != st[2]) ||
        (d_grad_x == d_grad_sum && st[0] != st[1]))
        return fail(SP_ERR_INVALID_ARG, "in place needs equal strides");
    if (d_grad_gain) {
        if (!d_workspace) return fail(SP_ERR_INVALID_ARG, "the gain's gradient needs a workspace");
        if (!aligned(d_workspace, 256)) return fail(SP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
        const size_t need = sp_norm_backward_workspace_bytes(dims);
        if (workspace_bytes < need) return fail(SP_ERR_INVALID_ARG, "workspace too small (%zu < %zu)", workspace_bytes, need);
    }
    if (dims->n_rows == 0) {
        const cudaError_t e = cudaMemsetAsync(d_grad_gain, 0, (size_t)dims->d * sizeof(float), (cudaStream_t)stream);
        return launched(e, "sp_norm_backward");
    }
    NormBackArgs a{dims->n_rows, dims->d, dims->dtype, dims->eps, st[0], st[1], st[2], st[3], d_grad_y, d_sum, d_grad_sum,
                   d_gain, d_grad_x, d_grad_gain, (float *)d_workspace};
    return launched(launch_norm_backward(a, sm_count(), (cudaStream_t)stream), "sp_norm_backward");
}

size_t sp_vocab_loss_workspace_bytes(const sp_vocab_dims *dims) {
    VocabArgs a;
    if (check_vocab(dims, false, &a) != SP_OK) return 0;
    return a.n ? lay_out(&a, false, nullptr) : 256;
}

sp_status sp_vocab_loss(sp_stream stream, const sp_vocab_dims *dims, const void *d_h, const void *d_w, const int *d_targets,
                        float *d_loss, float *d_lse, void *d_workspace, size_t workspace_bytes, int *d_status) {
    VocabArgs a;
    sp_status s = check_vocab(dims, false, &a);
    if (s != SP_OK || a.n == 0) return s;
    if (!d_loss || !d_lse) return fail(SP_ERR_INVALID_ARG, "a required pointer is NULL");
    s = check_vocab_buffers(&a, false, d_h, d_w, d_targets, nullptr, nullptr, d_lse, d_loss, d_workspace, workspace_bytes);
    if (s != SP_OK) return s;
    a.loss = d_loss;
    a.lse = d_lse;
    a.status = d_status;
    const cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = a.direct ? cudaSuccess : launch_vocab_keep(a, false, st);
    if (e == cudaSuccess) e = a.tensor ? launch_vocab_loss_tc(a, st) : launch_vocab_loss_simt(a, st);
    if (e == cudaSuccess) e = launch_vocab_finish_loss(a, st);
    return launched(e, "sp_vocab_loss");
}

size_t sp_vocab_loss_backward_workspace_bytes(const sp_vocab_dims *dims) {
    VocabArgs a;
    if (check_vocab(dims, true, &a) != SP_OK) return 0;
    return a.n ? lay_out(&a, true, nullptr) : 256;
}

sp_status sp_vocab_loss_backward(sp_stream stream, const sp_vocab_dims *dims, const void *d_h, const void *d_w,
                                 const int *d_targets, const float *d_lse, const float *d_grad_loss, void *d_grad_h,
                                 void *d_grad_w, void *d_workspace, size_t workspace_bytes, int *d_status) {
    VocabArgs a;
    sp_status s = check_vocab(dims, true, &a);
    if (s != SP_OK) return s;
    const cudaStream_t st = (cudaStream_t)stream;
    if (a.n == 0) {
        if (!d_grad_w) return SP_OK;
        const size_t es = elem_bytes(a.dtype);
        return launched(cudaMemset2DAsync(d_grad_w, (size_t)a.ws * es, 0, (size_t)a.d * es, (size_t)a.V, st), "sp_vocab_loss_backward");
    }
    if (!d_lse || !d_grad_h) return fail(SP_ERR_INVALID_ARG, "a required pointer is NULL");
    s = check_vocab_buffers(&a, true, d_h, d_w, d_targets, d_grad_h, d_grad_w, d_lse, d_grad_loss, d_workspace, workspace_bytes);
    if (s != SP_OK) return s;
    a.lse_in = d_lse;
    a.dloss = d_grad_loss;
    a.dh = d_grad_h;
    a.dw = d_grad_w;
    a.status = d_status;
    cudaError_t e = launch_vocab_keep(a, true, st);
    if (e == cudaSuccess) e = a.tensor ? launch_vocab_backward_tc(a, st) : launch_vocab_backward_simt(a, st);
    if (e == cudaSuccess) e = launch_vocab_finish_dh(a, st);
    return launched(e, "sp_vocab_loss_backward");
}

}  // extern "C"

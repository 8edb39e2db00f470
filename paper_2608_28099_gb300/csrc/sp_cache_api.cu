// C entry points of the token-cache operators: argument checks and launches.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <string.h>

#include "sp_cache.cuh"
#include "sp_gemm.cuh"

using namespace sp;

namespace {

sp_status fail(sp_status st, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    set_error_text(buf);
    return st;
}

sp_status launched(cudaError_t e, const char *what) {
    return e == cudaSuccess ? SP_OK : fail(SP_ERR_CUDA, "%s: launch failed: %s", what, cudaGetErrorString(e));
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// SMs of the current device, asked for once a device (a call's launch path).
int sm_count() {
    static int known[MAX_DEVICES] = {};
    int dev = 0, n = 152;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        cudaGetLastError();  // (no device: the host-only checks still answer)
        return n;
    }
    if (dev >= 0 && dev < MAX_DEVICES && known[dev]) return known[dev];
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && dev >= 0 && dev < MAX_DEVICES)
        known[dev] = n;
    return n;
}

// Whether any two of n x m blocks of `width` elements, a and b (>= width) apart, overlap.
bool blocks_overlap(long long n, long long a, long long m, long long b, long long width) {
    if (n < 2 || m < 2) return false;
    if (a > b) {
        const long long x = a, y = n;
        a = b, b = x, n = m, m = y;
    }
    for (long long j = 1; j < m; ++j) {  // blocks of the wider step, as far as those of the other reach
        const long long i = j * b / a, rest = j * b - i * a;
        if (i >= n) break;
        if (rest < width || (i + 1 < n && a - rest < width)) return true;
    }
    return false;
}

bool float_type(int dtype) { return dtype == SP_F32 || dtype == SP_BF16; }

sp_status check_rotary(const sp_rotary *r, RotaryDev *out) {
    if (!r) return fail(SP_ERR_INVALID_ARG, "rotary is NULL");
    if (r->head_dim < 1 || r->head_dim > 1024) return fail(SP_ERR_INVALID_ARG, "rotary head_dim must be in 1..1024");
    if (r->rot_dim < 2 || r->rot_dim > r->head_dim || r->rot_dim % 2)
        return fail(SP_ERR_INVALID_ARG, "rot_dim must be even and in 2..head_dim");
    if (r->interleaved != 0 && r->interleaved != 1) return fail(SP_ERR_INVALID_ARG, "interleaved must be 0 or 1");
    if (!isfinite(r->amplitude)) return fail(SP_ERR_INVALID_ARG, "amplitude must be finite");
    if (!r->d_turns) return fail(SP_ERR_INVALID_ARG, "rotary d_turns is NULL");
    *out = RotaryDev{r->rot_dim, r->rot_dim / 2, r->interleaved, r->amplitude, r->d_turns};
    return SP_OK;
}

sp_status check_cache(const sp_token_cache *c, CacheDev *out) {
    if (!c) return fail(SP_ERR_INVALID_ARG, "cache is NULL");
    const sp_kv_cache &kv = c->kv;
    if (!float_type(c->dtype) && c->dtype != SP_E4M3) return fail(SP_ERR_INVALID_ARG, "bad cache dtype %d", c->dtype);
    if (c->n_kv_heads < 1) return fail(SP_ERR_INVALID_ARG, "n_kv_heads must be >= 1");
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128)
        return fail(SP_ERR_UNSUPPORTED, "head_dim %d unsupported (32, 64, 128)", c->head_dim);
    // (a block's rows and a head's place in a row are 32-bit numbers in the kernels)
    if ((long long)c->n_kv_heads * c->head_dim > 0x7fffffffLL / 8) return fail(SP_ERR_UNSUPPORTED, "too many heads");
    if (c->max_seq_len < 0 || c->max_seq_len > 0x7fffffff - 4096)
        return fail(SP_ERR_INVALID_ARG, "max_seq_len out of range");
    if (kv.n_seqs < 1) return fail(SP_ERR_INVALID_ARG, "kv.n_seqs must be >= 1");
    if (kv.layout == SP_KV_CONTIGUOUS) {
        if (!kv.k_seq || !kv.v_seq) return fail(SP_ERR_INVALID_ARG, "a contiguous cache needs k_seq and v_seq");
    } else if (kv.layout == SP_KV_PAGED) {
        if (!kv.k_pool || !kv.v_pool || !kv.page_table)
            return fail(SP_ERR_INVALID_ARG, "a paged cache needs k_pool, v_pool and page_table");
        if ((((uintptr_t)kv.k_pool) | ((uintptr_t)kv.v_pool)) & 15)
            return fail(SP_ERR_INVALID_ARG, "k_pool and v_pool must be 16-byte aligned");
        if (kv.page_size != 16 && kv.page_size != 32 && kv.page_size != 64)
            return fail(SP_ERR_UNSUPPORTED, "page_size %d unsupported (16, 32, 64)", kv.page_size);
        if (kv.n_pages < 1 || kv.max_pages_per_seq < 1)
            return fail(SP_ERR_INVALID_ARG, "n_pages and max_pages_per_seq must be >= 1");
    } else {
        return fail(SP_ERR_INVALID_ARG, "bad kv layout %d", kv.layout);
    }
    if (c->dtype == SP_E4M3) {
        if (!c->k_scale || !c->v_scale) return fail(SP_ERR_INVALID_ARG, "an 8-bit cache needs k_scale and v_scale");
        if (kv.layout == SP_KV_PAGED && ((((uintptr_t)c->k_scale) | ((uintptr_t)c->v_scale)) & 15))
            return fail(SP_ERR_INVALID_ARG, "k_scale and v_scale must be 16-byte aligned");
    }
    out->kv = KVDev{kv.layout, kv.k_seq, kv.v_seq, kv.k_pool, kv.v_pool, kv.page_table, kv.page_size, kv.n_pages,
                    kv.max_pages_per_seq, kv.n_seqs};
    out->dtype = c->dtype;
    out->Hkv = c->n_kv_heads;
    out->dh = c->head_dim;
    out->max_seq_len = c->max_seq_len;
    out->k_scale = c->k_scale;
    out->v_scale = c->v_scale;
    return SP_OK;
}

// The common part of append and read.
sp_status check_copy(const sp_token_cache *cache, int batch, const int *d_seq_ids, const int *d_seq_lens,
                     const sp_token_rows *rows, int dtype, const void *d_k, const void *d_v, CopyArgs *a) {
    memset(a, 0, sizeof *a);
    sp_status s = check_cache(cache, &a->cache);
    if (s != SP_OK) return s;
    if (batch < 1) return fail(SP_ERR_INVALID_ARG, "batch must be >= 1");
    if (!rows) return fail(SP_ERR_INVALID_ARG, "rows is NULL");
    if (rows->max_rows < 1 || rows->n_rows < 1) return fail(SP_ERR_INVALID_ARG, "max_rows and n_rows must be >= 1");
    if ((long long)rows->max_rows * batch > 0x7fffffffLL)
        return fail(SP_ERR_UNSUPPORTED, "batch x max_rows above 2^31 - 1");
    if (!float_type(dtype)) return fail(SP_ERR_INVALID_ARG, "bad dtype %d of the rows", dtype);
    if (!d_seq_lens || !d_k || !d_v) return fail(SP_ERR_INVALID_ARG, "a required pointer is NULL");
    if (!d_seq_ids && batch > cache->kv.n_seqs)
        return fail(SP_ERR_INVALID_ARG, "batch %d exceeds n_seqs %d with implicit ids", batch, cache->kv.n_seqs);
    const long long dense = (long long)cache->n_kv_heads * cache->head_dim;
    const long long ks = rows->k_stride ? rows->k_stride : dense, vs = rows->v_stride ? rows->v_stride : dense;
    if (ks < dense || vs < dense) return fail(SP_ERR_INVALID_ARG, "k_stride and v_stride must be >= n_kv_heads * head_dim");
    const int es = dtype == SP_F32 ? 4 : 2;
    if ((((uintptr_t)d_k) | ((uintptr_t)d_v)) & (es - 1)) return fail(SP_ERR_INVALID_ARG, "rows must be aligned to their type");
    a->vec = !((((uintptr_t)d_k) | ((uintptr_t)d_v) | (uintptr_t)(ks * es) | (uintptr_t)(vs * es)) & 15);
    a->rows = RowsDev{rows->d_row0, rows->d_count, rows->d_take, rows->max_rows, rows->n_rows, ks, vs};
    a->B = batch;
    a->seq_ids = d_seq_ids;
    a->seq_lens = d_seq_lens;
    a->dtype = dtype;
    a->k = const_cast<void *>(d_k);
    a->v = const_cast<void *>(d_v);
    return SP_OK;
}

// Shapes of a tree call; fills what does not depend on the buffers.
sp_status check_tree(const sp_tree_dims *d, const sp_token_cache *cache, int batch, TreeArgs *a) {
    memset(a, 0, sizeof *a);
    if (!d) return fail(SP_ERR_INVALID_ARG, "dims is NULL");
    sp_status s = check_cache(cache, &a->cache);
    if (s != SP_OK) return s;
    if (batch < 1) return fail(SP_ERR_INVALID_ARG, "batch must be >= 1");
    if (batch > 65535) return fail(SP_ERR_UNSUPPORTED, "batch above 65535");
    const int Hkv = cache->n_kv_heads, dh = cache->head_dim;
    if (d->n_q_heads < 1 || d->n_q_heads % Hkv)
        return fail(SP_ERR_INVALID_ARG, "n_q_heads must be a positive multiple of n_kv_heads");
    if (d->n_nodes < 1 || d->n_nodes > 64) return fail(SP_ERR_INVALID_ARG, "n_nodes must be in 1..64");
    if (!float_type(d->dtype)) return fail(SP_ERR_INVALID_ARG, "bad dtype %d", d->dtype);
    if (d->path < 0 || d->path > 2) return fail(SP_ERR_INVALID_ARG, "bad path %d", d->path);
    if (d->shared_mask != 0 && d->shared_mask != 1) return fail(SP_ERR_INVALID_ARG, "shared_mask must be 0 or 1");
    if (!isfinite(d->scale) || d->scale < 0.f) return fail(SP_ERR_INVALID_ARG, "scale must be finite and >= 0");
    const long long rows = (long long)(d->n_q_heads / Hkv) * d->n_nodes;  // of a kv head
    if (Hkv * ceil_div_ll(rows, 32) > 65535) return fail(SP_ERR_UNSUPPORTED, "too many query rows");
    a->B = batch;
    a->Hq = d->n_q_heads;
    a->Hkv = Hkv;
    a->G = d->n_q_heads / Hkv;
    a->N = d->n_nodes;
    a->dh = dh;
    a->R = (int)rows;
    a->dtype = d->dtype;
    a->scale_log2 = (float)(1.4426950408889634 * (d->scale > 0.f ? (double)d->scale : 1.0 / sqrt((double)dh)));
    a->qs = d->q_stride ? d->q_stride : (long long)a->Hq * dh;
    a->ks = d->k_stride ? d->k_stride : (long long)Hkv * dh;
    a->vs = d->v_stride ? d->v_stride : (long long)Hkv * dh;
    if (a->qs < (long long)a->Hq * dh || a->ks < (long long)Hkv * dh || a->vs < (long long)Hkv * dh)
        return fail(SP_ERR_INVALID_ARG, "a node's row does not fit its stride");
    const int es = d->dtype == SP_F32 ? 4 : 2;
    if ((a->qs * es | a->ks * es | a->vs * es) & 15)
        return fail(SP_ERR_INVALID_ARG, "q_stride, k_stride and v_stride must be multiples of 16 bytes");
    a->mask_stride = d->shared_mask ? 0 : a->N;
    const long long paged = (long long)cache->kv.max_pages_per_seq * cache->kv.page_size;
    a->most_len = cache->kv.layout == SP_KV_PAGED && paged < cache->max_seq_len ? (int)paged : cache->max_seq_len;
    a->tensor = d->path != 1 && tree_tc_supported(*a);
    if (d->path == 2 && !a->tensor)
        return fail(SP_ERR_UNSUPPORTED, "the tensor-core kernel needs bf16 rows, a bf16 or 8-bit cache of head_dim 128 "
                                        "and a batch of at most 2048");
    if (a->tensor) plan_tree_tc(a, sm_count());
    else plan_tree_simt(a, sm_count());
    return SP_OK;
}

// Workspace: partials [slot][row][dh], their (max, sum), then the tensor-core kernel's
// table of shares (never nothing: 0 bytes answer an error).
size_t tree_rows(const TreeArgs &a) { return (a.tensor ? tree_tc_slots(a) : tree_simt_slots(a)) * a.rb_rows; }
size_t tree_o_bytes(const TreeArgs &a) { return align256(tree_rows(a) * a.dh * sizeof(float)); }
size_t tree_ml_bytes(const TreeArgs &a) { return align256(tree_rows(a) * 2 * sizeof(float)); }
size_t tree_bytes(const TreeArgs &a) {
    return tree_o_bytes(a) + tree_ml_bytes(a) + align256((size_t)(a.tensor ? tree_tc_groups(a) : 1) * sizeof(int2));
}

}  // namespace

extern "C" {

sp_status sp_rotary_plan(int kind, int rot_dim, double theta, double factor, double trained_len, double few,
                         double many, uint64_t *h_turns, float *amplitude) {
    if (!h_turns || !amplitude) return fail(SP_ERR_INVALID_ARG, "a required pointer is NULL");
    if (kind < SP_ROPE_PLAIN || kind > SP_ROPE_DIMS) return fail(SP_ERR_INVALID_ARG, "bad kind %d", kind);
    if (rot_dim < 2 || rot_dim > 1024 || rot_dim % 2) return fail(SP_ERR_INVALID_ARG, "rot_dim must be even and in 2..1024");
    if (!(theta > 1.0) || !isfinite(theta) || !(factor >= 1.0) || !isfinite(factor))
        return fail(SP_ERR_INVALID_ARG, "theta must be above 1 and factor at least 1");
    if (kind == SP_ROPE_BASE && rot_dim < 4) return fail(SP_ERR_INVALID_ARG, "SP_ROPE_BASE needs rot_dim >= 4");
    const bool ramp = kind == SP_ROPE_TURNS || kind == SP_ROPE_DIMS;
    if (ramp && !(trained_len > 0 && isfinite(trained_len) && few > 0 && many > few && isfinite(many)))
        return fail(SP_ERR_INVALID_ARG, "needs trained_len > 0 and 0 < few < many");
    const double tau = 6.283185307179586476925286766559;
    if (kind == SP_ROPE_BASE) theta *= pow(factor, rot_dim / (rot_dim - 2.0));
    // SP_ROPE_DIMS: the pairs with `many` and with `few` turns over trained_len
    const auto pair_at = [&](double n) { return 0.5 * rot_dim * log(trained_len / (tau * n)) / log(theta); };
    double lo = 0, hi = 0;
    if (kind == SP_ROPE_DIMS) {
        lo = fmax(floor(pair_at(many)), 0.0);
        hi = fmin(ceil(pair_at(few)), rot_dim - 1.0);
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(theta, -2.0 * i / rot_dim) / tau;  // turns a position
        if (kind == SP_ROPE_LINEAR) f /= factor;
        if (ramp) {
            const double w = kind == SP_ROPE_TURNS ? (trained_len * f - few) / (many - few)
                                                   : 1.0 - (i - lo) / fmax(hi - lo, 1e-3);
            const double keep = fmin(fmax(w, 0.0), 1.0);
            f = keep * f + (1.0 - keep) * f / factor;
        }
        h_turns[i] = (uint64_t)llrint(ldexp(f, 62)) << 2;  // (f < 1/2: fits)
    }
    *amplitude = kind == SP_ROPE_DIMS ? (float)(1.0 + 0.1 * log(factor)) : 1.f;
    return SP_OK;
}

sp_status sp_rotate(sp_stream stream, const sp_rotary *rot, int n_tokens, const int *d_positions, int backward,
                    int dtype, int n_heads, const void *d_x, long long x_token_stride, long long x_head_stride,
                    void *d_y, long long y_token_stride, long long y_head_stride) {
    RotateArgs a;
    memset(&a, 0, sizeof a);
    sp_status s = check_rotary(rot, &a.rot);
    if (s != SP_OK) return s;
    if (n_tokens < 0) return fail(SP_ERR_INVALID_ARG, "n_tokens must be >= 0");
    if (n_heads < 1) return fail(SP_ERR_INVALID_ARG, "n_heads must be >= 1");
    if ((long long)n_heads * rot->head_dim > 0x7fffffffLL / 8) return fail(SP_ERR_UNSUPPORTED, "too many heads");
    if (!float_type(dtype)) return fail(SP_ERR_INVALID_ARG, "bad dtype %d", dtype);
    if (backward != 0 && backward != 1) return fail(SP_ERR_INVALID_ARG, "backward must be 0 or 1");
    if (n_tokens == 0) return SP_OK;
    if (!d_positions || !d_x || !d_y) return fail(SP_ERR_INVALID_ARG, "a required pointer is NULL");
    const int es = dtype == SP_F32 ? 4 : 2;
    if ((((uintptr_t)d_x) | ((uintptr_t)d_y)) & (es - 1)) return fail(SP_ERR_INVALID_ARG, "x and y must be aligned to their type");
    if (x_token_stride < 0 || x_head_stride < 0 || y_token_stride < 0 || y_head_stride < 0)
        return fail(SP_ERR_INVALID_ARG, "strides must be >= 0");
    if ((n_heads > 1 && y_head_stride < rot->head_dim) || (n_tokens > 1 && y_token_stride < rot->head_dim) ||
        blocks_overlap(n_heads, y_head_stride, n_tokens, y_token_stride, rot->head_dim))
        return fail(SP_ERR_INVALID_ARG, "heads or tokens of y overlap");
    if (d_x == d_y && (x_token_stride != y_token_stride || x_head_stride != y_head_stride))
        return fail(SP_ERR_INVALID_ARG, "in place needs equal strides");
    a.n_tokens = n_tokens;
    a.n_heads = n_heads;
    a.dh = rot->head_dim;
    a.backward = backward;
    a.pos = d_positions;
    a.x = d_x;
    a.y = d_y;
    a.xt = x_token_stride;
    a.xh = x_head_stride;
    a.yt = y_token_stride;
    a.yh = y_head_stride;
    return launched(launch_rotate(dtype, a, sm_count(), (cudaStream_t)stream), "sp_rotate");
}

sp_status sp_cache_append(sp_stream stream, const sp_token_cache *cache, const sp_rotary *rot, int batch,
                          const int *d_seq_ids, const int *d_seq_lens, const sp_token_rows *rows, int dtype,
                          const void *d_k, const void *d_v, int *d_status) {
    CopyArgs a;
    sp_status s = check_copy(cache, batch, d_seq_ids, d_seq_lens, rows, dtype, d_k, d_v, &a);
    if (s != SP_OK) return s;
    if (rot) {
        s = check_rotary(rot, &a.rot);
        if (s != SP_OK) return s;
        if (rot->head_dim != cache->head_dim)
            return fail(SP_ERR_INVALID_ARG, "rotary head_dim %d, cache head_dim %d", rot->head_dim, cache->head_dim);
    }
    a.status = d_status;
    return launched(launch_append(a, sm_count(), (cudaStream_t)stream), "sp_cache_append");
}

sp_status sp_cache_read(sp_stream stream, const sp_token_cache *cache, int batch, const int *d_seq_ids,
                        const int *d_seq_lens, const int *d_first, const sp_token_rows *rows, int dtype, void *d_k,
                        void *d_v, int *d_status) {
    CopyArgs a;
    sp_status s = check_copy(cache, batch, d_seq_ids, d_seq_lens, rows, dtype, d_k, d_v, &a);
    if (s != SP_OK) return s;
    a.first = d_first;
    a.status = d_status;
    return launched(launch_read(a, sm_count(), (cudaStream_t)stream), "sp_cache_read");
}

sp_status sp_tree_masks(int n_nodes, const int *h_parent, uint64_t *h_mask, int *h_depth) {
    if (n_nodes < 1 || n_nodes > 64) return fail(SP_ERR_INVALID_ARG, "n_nodes must be in 1..64");
    if (!h_parent || !h_mask) return fail(SP_ERR_INVALID_ARG, "a required pointer is NULL");
    for (int i = 0; i < n_nodes; ++i)
        if (h_parent[i] < -1 || h_parent[i] >= i)
            return fail(SP_ERR_INVALID_ARG, "parent of node %d is %d, neither -1 nor an earlier node", i, h_parent[i]);
    int depth[64];
    for (int i = 0; i < n_nodes; ++i) {
        const int p = h_parent[i];
        h_mask[i] = (1ull << i) | (p >= 0 ? h_mask[p] : 0);
        depth[i] = p >= 0 ? depth[p] + 1 : 0;
    }
    if (h_depth) memcpy(h_depth, depth, n_nodes * sizeof(int));
    return SP_OK;
}

size_t sp_attend_tree_workspace_bytes(const sp_tree_dims *dims, const sp_token_cache *cache, int batch) {
    TreeArgs a;
    return check_tree(dims, cache, batch, &a) == SP_OK ? tree_bytes(a) : 0;
}

sp_status sp_attend_tree(sp_stream stream, const sp_tree_dims *dims, const sp_token_cache *cache, int batch,
                         const int *d_seq_ids, const int *d_seq_lens, const uint64_t *d_mask, const int *d_n_nodes,
                         const void *d_q, const void *d_k_new, const void *d_v_new, void *d_out, void *d_workspace,
                         size_t workspace_bytes, int *d_status) {
    TreeArgs a;
    sp_status s = check_tree(dims, cache, batch, &a);
    if (s != SP_OK) return s;
    if (!d_seq_lens || !d_q || !d_k_new || !d_v_new || !d_out || !d_workspace)
        return fail(SP_ERR_INVALID_ARG, "a required pointer is NULL");
    if (!d_seq_ids && batch > cache->kv.n_seqs)
        return fail(SP_ERR_INVALID_ARG, "batch %d exceeds n_seqs %d with implicit ids", batch, cache->kv.n_seqs);
    if (((uintptr_t)d_workspace) & 255) return fail(SP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if ((((uintptr_t)d_q) | ((uintptr_t)d_k_new) | ((uintptr_t)d_v_new) | ((uintptr_t)d_out)) & 15)
        return fail(SP_ERR_INVALID_ARG, "queries, new keys/values and the output must be 16-byte aligned");
    const size_t need = tree_bytes(a);
    if (workspace_bytes < need) return fail(SP_ERR_INVALID_ARG, "workspace too small (%zu < %zu)", workspace_bytes, need);
    a.seq_ids = d_seq_ids;
    a.seq_lens = d_seq_lens;
    a.n_nodes = d_n_nodes;
    a.mask = d_mask;
    a.q = d_q;
    a.k_new = d_k_new;
    a.v_new = d_v_new;
    a.out = d_out;
    a.part_o = (float *)d_workspace;
    a.part_ml = (float *)((char *)d_workspace + tree_o_bytes(a));
    a.status = d_status;
    int2 *split_tab = (int2 *)((char *)a.part_ml + tree_ml_bytes(a));
    return launched(a.tensor ? launch_tree_tc(a, split_tab, (cudaStream_t)stream) : launch_tree_simt(a, (cudaStream_t)stream),
                    "sp_attend_tree");
}

}  // extern "C"

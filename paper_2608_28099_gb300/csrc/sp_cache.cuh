// Internal declarations of the token-cache operators: rotary positions, appending
// to and reading from a cache, and the attention of a drafted tree.
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "sp_common.cuh"

namespace sp {

// Smallest amax that a token's 8-bit scale is made of: 448 / it and its product with
// any code stay far from the ends of fp32, and log2 of the scale is finite.
constexpr float kMinAmax = 8.673617379884035e-19f;  // 2^-60
constexpr float kMaxCode = 448.f;                   // the largest 8-bit value
constexpr float kLeastWeight = 1.401298464324817e-45f;  // 2^-149, where a weight that a row sees would be 0

// A cache as the kernels see it.
struct CacheDev {
    KVDev kv;
    int dtype, Hkv, dh, max_seq_len;
    void *k_scale, *v_scale;
};

struct RotaryDev {
    int rot, half, interleaved;  // rotated dims, pairs, layout
    float amplitude;
    const uint64_t *turns;
};

struct RowsDev {
    const int *row0, *count, *take;
    int max_rows, n_rows;
    long long k_stride, v_stride;  // elements
};

// cos and sin (times the amplitude) of pair i at position pos: the phase is a wrapping
// 64-bit product, its top 32 bits a signed fraction of a turn (2^-32 turn), so the
// error does not grow with the position.
__device__ __forceinline__ float2 rotary_cs(const RotaryDev &r, int pos, int i) {
    const uint64_t ph = (uint64_t)(long long)pos * r.turns[i];
    float s, c;
    sincospif((float)(int)(ph >> 32) * 4.656612873077393e-10f, &s, &c);  // 2^-31: half turns
    return make_float2(c * r.amplitude, s * r.amplitude);
}

// Where token t of a resolved sequence sits: the index of its (token, head 0) row in
// units of (token, kv head) rows, and the step from a head to the next; false if it
// has no page.  Paged: of the pool; contiguous: of the sequence's own buffer.
__device__ __forceinline__ bool cache_row(const CacheDev &c, int sid, int t, long long *row, int *head_step) {
    if (c.kv.layout == SP_KV_PAGED) {
        const int P = c.kv.page_size, lp = t / P;
        const int page = lp < c.kv.max_pages ? c.kv.page_table[(size_t)sid * c.kv.max_pages + lp] : -1;
        if (page < 0 || page >= c.kv.n_pages) return false;
        *row = (long long)page * c.Hkv * P + (t - lp * P);
        *head_step = P;
    } else {
        *row = (long long)t * c.Hkv;
        *head_step = 1;
    }
    return true;
}
__device__ __forceinline__ void *cache_base(const CacheDev &c, int sid, int is_v) {
    if (c.kv.layout == SP_KV_PAGED) return const_cast<void *>(is_v ? c.kv.v_pool : c.kv.k_pool);
    return const_cast<void *>((is_v ? c.kv.v_seq : c.kv.k_seq)[sid]);
}
__device__ __forceinline__ float *scale_base(const CacheDev &c, int sid, int is_v) {
    void *p = is_v ? c.v_scale : c.k_scale;
    return c.kv.layout == SP_KV_PAGED ? (float *)p : ((float *const *)p)[sid];
}

// 8 codes (little-endian bytes) as floats, unscaled.
__device__ __forceinline__ void codes_to_float(uint2 u, float (&v)[8]) {
    const uint32_t w[2] = {u.x, u.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ uint32_t float_to_codes2(float a, float b) {
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// ---------------------------------------------------------------------------
struct RotateArgs {
    RotaryDev rot;
    int n_tokens, n_heads, dh, backward;
    const int *pos;
    const void *x;
    void *y;
    long long xt, xh, yt, yh;  // strides, elements
    int tokens_per_block, groups;  // (set by the launch)
};
cudaError_t launch_rotate(int dtype, const RotateArgs &a, int n_sm, cudaStream_t st);

struct CopyArgs {  // append (rows -> cache) and read (cache -> rows)
    CacheDev cache;
    RotaryDev rot;             // append: rot.rot = 0 without a rotation
    RowsDev rows;
    int B;
    const int *seq_ids, *seq_lens, *first;
    int dtype;                 // of the rows
    void *k, *v;
    int vec;                   // rows in 16-byte vectors
    int tokens_per_block, chunks;  // blocks a sequence (set by the launch)
    int *status;
};
cudaError_t launch_append(const CopyArgs &a, int n_sm, cudaStream_t st);
cudaError_t launch_read(const CopyArgs &a, int n_sm, cudaStream_t st);

// ---------------------------------------------------------------------------
struct TreeArgs {
    CacheDev cache;
    int B, Hq, Hkv, G, N, dh;      // N: most nodes
    int R;                         // G N query rows of a kv head: row rr = node G + head of the group
    int n_rb, rb_rows;             // row blocks of a kv head and the rows of each (the last has fewer)
    int dtype;                     // of q, k_new, v_new, out
    bool tensor;                   // which kernel
    float scale_log2;              // log2(e) * scale of the scores
    // Most cached tokens of a sequence: max_seq_len, or what the page table has room for.
    // max_seq_len may be no bound at all, and a corrupt length would then keep a kernel at it for
    // seconds, with tile numbers of more than 31 bits.
    int most_len;
    const int *seq_ids, *seq_lens, *n_nodes;
    const uint64_t *mask;          // NULL: a chain
    int mask_stride;               // words from a sequence to the next (0: shared)
    const void *q, *k_new, *v_new;
    long long qs, ks, vs;          // elements from a node's row to the next
    void *out;
    float *lse;                    // NULL, or [B N][Hq]: log of the sum of a row's exponentials
    int n_splits, split_tokens;    // CUDA cores: shares of a sequence's [cache ; tree]
    AttnArgs plan;                 // tensor cores: what sp_attn_plan.cuh cuts the work by
    float *part_o, *part_ml;       // [slot][rb_rows][dh] unnormalised, [slot][rb_rows][2] (max in
                                   // log2 units, sum)
    int *status;
};

__device__ __forceinline__ int checked_nodes(const TreeArgs &a, int n, int *status) {
    if (n < 0 || n > a.N) {
        if (status) atomicOr(status, SP_DEV_BAD_ROW);
        n = n < 0 ? 0 : a.N;
    }
    return n;
}
__device__ __forceinline__ int tree_nodes(const TreeArgs &a, int b, int *status) {
    return checked_nodes(a, a.n_nodes ? a.n_nodes[b] : a.N, status);
}
// log of a row's sum of exponentials from its (max in log2 units, sum); -inf: it sees nothing.
__device__ __forceinline__ void store_lse(const TreeArgs &a, int b, int node, int head, float m, float l) {
    a.lse[((size_t)b * a.N + node) * a.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
}
// The nodes that node i of sequence b sees.
__device__ __forceinline__ uint64_t tree_mask(const TreeArgs &a, int b, int i, int n) {
    const uint64_t all = n >= 64 ? ~0ull : (1ull << n) - 1;
    return (a.mask ? a.mask[(size_t)b * a.mask_stride + i] : (2ull << i) - 1) & all;
}

// Lets a kernel take `bytes` of dynamic shared memory on the current device.  The calls have no
// handle that would tie them to one, and the limit is each device's own: asked for once a device
// (known: the kernel's).
constexpr int MAX_DEVICES = 64;
template <typename Kern>
inline cudaError_t allow_smem(Kern kernel, int bytes, bool (&known)[MAX_DEVICES]) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < MAX_DEVICES && known[dev])) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < MAX_DEVICES) known[dev] = true;
    return e;
}
// CUDA cores: every shape, fp32 arithmetic; shares of a sequence merged by a second kernel.
void plan_tree_simt(TreeArgs *a, int n_sm);
cudaError_t launch_tree_simt(const TreeArgs &a, cudaStream_t st);
size_t tree_simt_slots(const TreeArgs &a);
// tcgen05: head_dim 128, bf16 rows, bf16 or 8-bit caches, B <= 2048; two launches.
// split_tab: tree_tc_groups int2 of scratch.
bool tree_tc_supported(const TreeArgs &a);
void plan_tree_tc(TreeArgs *a, int n_sm);
size_t tree_tc_slots(const TreeArgs &a);
int tree_tc_groups(const TreeArgs &a);
cudaError_t launch_tree_tc(const TreeArgs &a, int2 *split_tab, cudaStream_t st);

// The backward pass (sp_tree_back.cu): TreeArgs with `out` the forward pass's output and `lse` its
// log sums, both read.
struct TreeBackArgs {
    TreeArgs t;
    const void *dout;
    void *dq, *dk, *dv;            // rows qs, ks, vs elements apart
    float2 *stat;                  // [B][Hkv][R]: (log sum in log2 units, +inf for a row that sees
                                   // nothing; sum of out * dout)
    float *dq_new;                 // [B][Hkv][R][dh]: the nodes' own part of dq, unscaled
    float scale;
};
// Row statistics, gradients of the nodes' keys and values and the nodes' part of dq; then the cache's
// part of dq in shares (t.part_o: [slot][row][dh]), and the sum of all parts.  CUDA cores:
cudaError_t launch_tree_back_simt(const TreeBackArgs &a, cudaStream_t st);
size_t tree_back_simt_slots(const TreeArgs &a);
// Tensor cores: head_dim 128, bf16 rows and cache, B <= 2048.
bool tree_back_tc_supported(const TreeArgs &a);
void plan_tree_back_tc(TreeArgs *a, int n_sm);
size_t tree_back_tc_slots(const TreeArgs &a);
int tree_back_tc_groups(const TreeArgs &a);
cudaError_t launch_tree_back_tc(const TreeBackArgs &a, int2 *split_tab, cudaStream_t st);
// What is not the cache's, by a kernel of its own: bf16 rows of 128 dims.
cudaError_t launch_tree_back_rows_tc(const TreeBackArgs &a, cudaStream_t st);

}  // namespace sp

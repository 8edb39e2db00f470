// Attention of a drafted tree over [cache ; tree] (Eq. 1-3, the causal part replaced
// by the tree's masks) on CUDA cores: every head_dim, type and layout, in fp32.  The
// kernel of fp32 callers (no tensor product keeps 24 bits) and of the shapes that the
// tensor-core kernel (sp_tree_tc.cu) does not take.
//
// A block takes 32 query rows of a (sequence, kv head) and a share of the tokens:
// tiles of 32 tokens, decoded to fp32 in shared memory, a token a lane for the scores,
// dh / 32 dims a lane for the values; a warp owns four rows with their running (max,
// sum, O).  Shares are merged by a second kernel.  Bound by shared-memory reads (5
// vector loads per 16 multiply-adds a lane in the score product).  Five sequences of 0 to 500
// tokens, 11 nodes, head_dim 32, fp32: 17 us with the merge, latency; eight of 1000 to 4000, 16
// nodes, 16 heads of 128, fp32: 180 us, 16 TFLOP/s.  Where the tensor-core kernel applies this
// one is not taken: one sequence of 2048 tokens, 8 nodes, 33 against 16 us; 64 tokens, one node,
// 18 against 12; 64 sequences of 1024 to 8192 tokens, 16 nodes, 4315 against 190 (an empty cache
// alone is faster here, 8.3 against 11.0, and lengths are not known to the host).  Those 64
// sequences with heads of 64 (32) dims, which that kernel does not take: 2990 (2035) us.
#include "sp_cache.cuh"
#include "sp_sm100.cuh"

namespace sp {

namespace {

constexpr int THREADS = 256;
constexpr int ROWS = 32;        // rows of a block
constexpr int RW = 4;           // rows of a warp
constexpr int TOK = 32;         // tokens of a tile

template <int DH>
struct Smem {
    float q[ROWS][DH];
    float k[TOK][DH + 4];       // (a token a lane: rows 4 banks apart)
    float v[TOK][DH];
};

// A weight, never 0: what vanishes beside the maximum still hands on a NaN or an infinity (2^-149 of
// a finite value adds nothing).
__device__ __forceinline__ float some_exp2(float x) {
    const float y = exp2f(x);
    return y == 0.f ? kLeastWeight : y;
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

__device__ __forceinline__ void load_elems(const void *p, int dtype, size_t e, float (&v)[8]) {
    if (dtype == SP_F32) load8((const float *)p + e, v);
    else load8((const bf16 *)p + e, v);
}

template <int DH>
__global__ void __launch_bounds__(THREADS) tree_simt_kernel(const __grid_constant__ TreeArgs a) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Smem<DH> &s = *(Smem<DH> *)smem_raw;
    constexpr int C = DH / 8, D = DH / 32;  // 8-element chunks of a row, dims a lane
    pdl_wait();
    pdl_trigger();
    const int hv = blockIdx.y, g = hv / a.n_rb, rb = hv - g * a.n_rb, b = blockIdx.z, split = blockIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int *status = threadIdx.x == 0 && hv == 0 && split == 0 ? a.status : nullptr;
    const SeqRef sq = resolve_seq(a.seq_ids, a.seq_lens, 0, b, a.cache.kv.n_seqs, a.most_len, status);
    const int n = tree_nodes(a, b, status), total = sq.len + n;
    const int t_lo = min(total, split * a.split_tokens), t_hi = t_lo + min(a.split_tokens, total - t_lo);
    const int row0 = rb * a.rb_rows;

    for (int i = threadIdx.x; i < ROWS * C; i += THREADS) {
        const int r = i / C, e = (i - r * C) * 8, rr = row0 + r, node = rr / a.G;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (rr < a.R && node < n)
            load_elems(a.q, a.dtype, (size_t)((size_t)b * a.N + node) * a.qs + (size_t)(g * a.G + rr - node * a.G) * DH + e, v);
#pragma unroll
        for (int x = 0; x < 8; ++x) s.q[r][e + x] = v[x] * a.scale_log2;
    }
    float m[RW], l[RW], o[RW][D];
    uint64_t sees[RW];
    bool live[RW];
#pragma unroll
    for (int r = 0; r < RW; ++r) {
        const int rr = row0 + warp * RW + r, node = rr / a.G;
        live[r] = rr < a.R && node < n;
        sees[r] = live[r] ? tree_mask(a, b, node, n) : 0;
        m[r] = -INFINITY;
        l[r] = 0.f;
#pragma unroll
        for (int d = 0; d < D; ++d) o[r][d] = 0.f;
    }
    bool bad = false;
    for (int t0 = t_lo; t0 < t_hi; t0 += TOK) {
        __syncthreads();
        for (int i = threadIdx.x; i < TOK * C; i += THREADS) {
            const int tt = i / C, e = (i - tt * C) * 8, t = t0 + tt;
            float k[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (t < t_hi && t < sq.len) {
                long long row;
                int step;
                if (cache_row(a.cache, sq.sid, t, &row, &step)) {
                    row += (long long)g * step;
                    const void *kb = cache_base(a.cache, sq.sid, 0), *vb = cache_base(a.cache, sq.sid, 1);
                    if (a.cache.dtype == SP_E4M3) {
                        codes_to_float(*(const uint2 *)((const uint8_t *)kb + row * DH + e), k);
                        codes_to_float(*(const uint2 *)((const uint8_t *)vb + row * DH + e), v);
                        const float fk = scale_base(a.cache, sq.sid, 0)[row], fv = scale_base(a.cache, sq.sid, 1)[row];
#pragma unroll
                        for (int x = 0; x < 8; ++x) k[x] *= fk, v[x] *= fv;
                    } else {
                        load_elems(kb, a.cache.dtype, (size_t)row * DH + e, k);
                        load_elems(vb, a.cache.dtype, (size_t)row * DH + e, v);
                    }
                } else {
                    bad = true;
                }
            } else if (t < t_hi) {
                const size_t r = (size_t)b * a.N + (t - sq.len);
                load_elems(a.k_new, a.dtype, r * a.ks + (size_t)g * DH + e, k);
                load_elems(a.v_new, a.dtype, r * a.vs + (size_t)g * DH + e, v);
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) s.k[tt][e + x] = k[x], s.v[tt][e + x] = v[x];
        }
        __syncthreads();
        float sc[RW] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int d = 0; d < DH; d += 4) {
            const float4 k = *(const float4 *)&s.k[lane][d];
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                const float4 q = *(const float4 *)&s.q[warp * RW + r][d];
                sc[r] += q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
            }
        }
        const int t = t0 + lane, j = t - sq.len;
#pragma unroll
        for (int r = 0; r < RW; ++r) {
            const bool visible = live[r] && t < t_hi && (j < 0 || ((sees[r] >> j) & 1));
            const float x = visible ? sc[r] : -INFINITY;
            const float mn = fmaxf(m[r], warp_max(x));
            // (a NaN score is not a maximum: it makes its own weight, and so the row, NaN)
            const float mu = mn == -INFINITY ? 0.f : mn;
            const float al = m[r] == -INFINITY ? 0.f : some_exp2(m[r] - mu);
            sc[r] = visible ? x == -INFINITY ? 0.f : some_exp2(x - mu) : 0.f;
            l[r] = l[r] * al + warp_sum(sc[r]);
            m[r] = mn;
#pragma unroll
            for (int d = 0; d < D; ++d) o[r][d] *= al;
        }
        // a weight of 0 is skipped: what a row does not see (NaN, infinities) must not
        // reach it as 0 * v (what it sees has at least the least weight)
#pragma unroll 4
        for (int x = 0; x < TOK; ++x) {
            float v[D];
#pragma unroll
            for (int d = 0; d < D; ++d) v[d] = s.v[x][lane + 32 * d];
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                const float p = __shfl_sync(0xffffffffu, sc[r], x);
                if (p != 0.f) {
#pragma unroll
                    for (int d = 0; d < D; ++d) o[r][d] += p * v[d];
                }
            }
        }
    }
    if (bad && a.status) atomicOr(a.status, SP_DEV_BAD_PAGE);
#pragma unroll
    for (int r = 0; r < RW; ++r) {
        const int local = warp * RW + r, rr = row0 + local;
        if (rr >= a.R) continue;
        if (a.n_splits == 1) {
            const int node = rr / a.G;
            const size_t at = ((size_t)b * a.N + node) * a.Hq * DH + (size_t)(g * a.G + rr - node * a.G) * DH;
#pragma unroll
            for (int d = 0; d < D; ++d) {
                const float y = live[r] && !(l[r] == 0.f) ? o[r][d] / l[r] : 0.f;
                if (a.dtype == SP_F32) ((float *)a.out)[at + lane + 32 * d] = y;
                else ((bf16 *)a.out)[at + lane + 32 * d] = __float2bfloat16_rn(y);
            }
            if (a.lse && lane == 0) store_lse(a, b, node, g * a.G + rr - node * a.G, m[r], live[r] ? l[r] : 0.f);
        } else {
            const size_t slot = ((size_t)b * gridDim.y + hv) * a.n_splits + split, row = slot * a.rb_rows + local;
#pragma unroll
            for (int d = 0; d < D; ++d) a.part_o[row * DH + lane + 32 * d] = o[r][d];
            if (lane == 0) *(float2 *)(a.part_ml + row * 2) = make_float2(m[r], l[r]);
        }
    }
}

// Merge of the shares: a warp per (sequence, kv head, row), in share order.
template <int DH>
__global__ void __launch_bounds__(THREADS) tree_merge_kernel(const __grid_constant__ TreeArgs a) {
    constexpr int D = DH / 32;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5);
    if (w >= (long long)a.B * a.Hkv * a.R) return;
    const int rr = (int)(w % a.R), g = (int)(w / a.R % a.Hkv), b = (int)(w / a.R / a.Hkv);
    const int rb = rr / a.rb_rows, hv = g * a.n_rb + rb;
    const size_t row0 = (((size_t)b * a.Hkv * a.n_rb + hv) * a.n_splits) * a.rb_rows + (rr - rb * a.rb_rows);
    float m = -INFINITY, l = 0.f, o[D];
#pragma unroll
    for (int d = 0; d < D; ++d) o[d] = 0.f;
    for (int s = 0; s < a.n_splits; ++s) {
        const size_t row = row0 + (size_t)s * a.rb_rows;
        const float2 ml = *(const float2 *)(a.part_ml + row * 2);
        const float mn = fmaxf(m, ml.x);
        if (ml.y == 0.f && ml.x == -INFINITY) continue;
        const float mu = mn == -INFINITY ? 0.f : mn;
        const float al = m == -INFINITY ? 0.f : some_exp2(m - mu), be = ml.x == -INFINITY ? 1.f : some_exp2(ml.x - mu);
        l = l * al + ml.y * be;
#pragma unroll
        for (int d = 0; d < D; ++d) o[d] = o[d] * al + a.part_o[row * DH + lane + 32 * d] * be;
        m = mn;
    }
    const int node = rr / a.G;
    const bool live = node < tree_nodes(a, b, nullptr) && !(l == 0.f);
    const size_t at = ((size_t)b * a.N + node) * a.Hq * DH + (size_t)(g * a.G + rr - node * a.G) * DH;
#pragma unroll
    for (int d = 0; d < D; ++d) {
        const float y = live ? o[d] / l : 0.f;
        if (a.dtype == SP_F32) ((float *)a.out)[at + lane + 32 * d] = y;
        else ((bf16 *)a.out)[at + lane + 32 * d] = __float2bfloat16_rn(y);
    }
    if (a.lse && lane == 0) store_lse(a, b, node, g * a.G + rr - node * a.G, m, live ? l : 0.f);
}

template <int DH>
cudaError_t run(const TreeArgs &a, cudaStream_t st) {
    static bool known[MAX_DEVICES] = {};
    cudaError_t e = allow_smem(tree_simt_kernel<DH>, (int)sizeof(Smem<DH>), known);
    if (e != cudaSuccess) return e;
    const dim3 grid(a.n_splits, a.Hkv * a.n_rb, a.B);
    e = launch_k(tree_simt_kernel<DH>, grid, dim3(THREADS), sizeof(Smem<DH>), st, a);
    if (e != cudaSuccess || a.n_splits == 1) return e;
    const long long rows = (long long)a.B * a.Hkv * a.R;
    return launch_k(tree_merge_kernel<DH>, dim3((unsigned)ceil_div_ll(rows, THREADS / 32)), dim3(THREADS), 0, st, a);
}

}  // namespace

// Row blocks of 32, and shares of at least 128 tokens until four blocks an SM.
void plan_tree_simt(TreeArgs *a, int n_sm) {
    a->rb_rows = ROWS;
    a->n_rb = ceil_div(a->R, ROWS);
    const int longest = a->cache.max_seq_len + a->N;
    const long long units = (long long)a->B * a->Hkv * a->n_rb;
    long long splits = (4ll * n_sm + units - 1) / units;
    splits = splits < 1 ? 1 : splits;
    const int most = ceil_div(longest, 128);
    if (splits > most) splits = most;
    a->split_tokens = ceil_div(ceil_div(longest, (int)splits), TOK) * TOK;
    a->n_splits = (longest - 1) / a->split_tokens + 1;  // (their sum may pass 31 bits)
}

size_t tree_simt_slots(const TreeArgs &a) {
    return a.n_splits == 1 ? 0 : (size_t)a.B * a.Hkv * a.n_rb * a.n_splits;
}

cudaError_t launch_tree_simt(const TreeArgs &a, cudaStream_t st) {
    if (a.dh == 128) return run<128>(a, st);
    if (a.dh == 64) return run<64>(a, st);
    return run<32>(a, st);
}

}  // namespace sp

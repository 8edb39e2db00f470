// Backward pass of the attention of a tree (or of a probe's soft-prompt rows) over [cache ; tree],
// the cache a constant.  With the forward pass's output o and log sums lse, for row r and token t:
//   p = exp(scale q.k - lse),  D = dout.o,  ds = p (dout.v - D)
//   dq_r = scale sum_t ds k_t,   dk_j = scale sum_r ds q_r,   dv_j = sum_r p dout_r   (nodes j)
// The log sums make every weight final where it is formed: parts of dq are sums, and nothing has to
// be rescaled or merged by a maximum.  Here: the row statistics and everything between the nodes (a
// block a (sequence, kv head), whose rows it takes 32 at a time with the nodes' gradients in
// registers, so that heads that share a kv head are added in one order), and the cache's part on
// CUDA cores in fp32 for the shapes and types that the tensor-core kernel does not take.  Bound by
// shared-memory reads, as the forward kernel is: 64 sequences of 1024 to 8192 tokens, 16 rows, heads of
// 128 bf16 dims 5475 us (214 on tensor cores), 17 to 20 TFLOP/s.
#include "sp_cache.cuh"

namespace sp {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;
constexpr int ROWS = 32, RW = ROWS / WARPS;  // rows of a tile, of a warp
constexpr int TOK = 32;                      // cached tokens of a tile
constexpr int MAX_N = 64;                    // nodes

template <int DH>
struct RowSmem {
    float k[MAX_N][DH + 4], v[MAX_N][DH + 4];  // (a node a lane: rows 4 banks apart)
    float q[ROWS][DH], dout[ROWS][DH];
    float p[ROWS][MAX_N], ds[ROWS][MAX_N];
    uint64_t sees[ROWS];
};
template <int DH, int TW>
struct CacheSmem {
    float k[TOK * TW][DH + 4], v[TOK * TW][DH + 4];
    float q[ROWS / TW][DH], dout[ROWS / TW][DH];
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
__device__ __forceinline__ void load_elems(const void *p, int dtype, size_t e, float (&v)[8]) {
    if (dtype == SP_F32) load8((const float *)p + e, v);
    else load8((const bf16 *)p + e, v);
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
    *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
    *(float4 *)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store_elem(void *p, int dtype, size_t e, float v) {
    if (dtype == SP_F32) ((float *)p)[e] = v;
    else ((bf16 *)p)[e] = __float2bfloat16_rn(v);
}
// Element where row rr of kv head g of sequence b starts, in rows `stride` elements apart.
__device__ __forceinline__ size_t row_at(const TreeArgs &a, int b, int g, int rr, long long stride) {
    const int node = rr / a.G;
    return ((size_t)b * a.N + node) * stride + (size_t)(g * a.G + rr - node * a.G) * a.dh;
}

// ---------------------------------------------------------------------------
template <int DH>
__global__ void __launch_bounds__(THREADS) tree_back_rows_kernel(const __grid_constant__ TreeBackArgs args) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    RowSmem<DH> &s = *(RowSmem<DH> *)smem_raw;
    const TreeArgs &a = args.t;
    constexpr int C = DH / 8, D = DH / 32;
    constexpr int NW = MAX_N / WARPS;  // nodes of a warp: dk, dv of lane + 32 d
    pdl_wait();
    pdl_trigger();
    const int g = blockIdx.x, b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int *status = threadIdx.x == 0 && g == 0 ? a.status : nullptr;
    const int n = tree_nodes(a, b, status);
    for (int i = threadIdx.x; i < MAX_N * C; i += THREADS) {
        const int j = i / C, e = (i - j * C) * 8;
        float k[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (j < n) {
            const size_t r = (size_t)b * a.N + j;
            load_elems(a.k_new, a.dtype, r * a.ks + (size_t)g * DH + e, k);
            load_elems(a.v_new, a.dtype, r * a.vs + (size_t)g * DH + e, v);
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) s.k[j][e + x] = k[x], s.v[j][e + x] = v[x];
    }
    float dk[NW][D], dv[NW][D];
#pragma unroll
    for (int j = 0; j < NW; ++j)
#pragma unroll
        for (int d = 0; d < D; ++d) dk[j][d] = dv[j][d] = 0.f;
    const size_t row0 = ((size_t)b * a.Hkv + g) * a.R;
    for (int r0 = 0; r0 < a.R; r0 += ROWS) {
        __syncthreads();
#pragma unroll 1
        for (int r = warp * RW; r < warp * RW + RW; ++r) {  // queries, output gradients, statistics
            const int rr = r0 + r, node = rr / a.G;
            const bool live = rr < a.R && node < n;
            float delta = 0.f;
#pragma unroll
            for (int d = 0; d < D; ++d) {
                const int e = lane + 32 * d;
                float q = 0.f, go = 0.f, o = 0.f;
                if (live) {
                    const size_t at = row_at(a, b, g, rr, (long long)a.Hq * DH) + e;
                    if (a.dtype == SP_F32) {
                        q = ((const float *)a.q)[row_at(a, b, g, rr, a.qs) + e];
                        go = ((const float *)args.dout)[at], o = ((const float *)a.out)[at];
                    } else {
                        q = to_f(((const bf16 *)a.q)[row_at(a, b, g, rr, a.qs) + e]);
                        go = to_f(((const bf16 *)args.dout)[at]), o = to_f(((const bf16 *)a.out)[at]);
                    }
                }
                s.q[r][e] = q, s.dout[r][e] = go;
                delta += go * o;
            }
            delta = warp_sum(delta);
            float l2 = INFINITY;
            if (live) {
                const float lse = a.lse[((size_t)b * a.N + node) * a.Hq + g * a.G + rr - node * a.G];
                if (lse != -INFINITY) l2 = lse == INFINITY ? NAN : lse * 1.4426950408889634f;
            }
            if (lane == 0) {
                s.sees[r] = l2 == INFINITY ? 0 : tree_mask(a, b, node, n);
                if (rr < a.R) args.stat[row0 + rr] = make_float2(l2, l2 == INFINITY ? 0.f : delta);
            }
            // weights and their gradients: two nodes a lane
            __syncwarp();
            const uint64_t sees = s.sees[r];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = lane + 32 * h;
                float x = 0.f, dp = 0.f;
                if (__any_sync(0xffffffffu, (sees >> j) & 1)) {
#pragma unroll 4
                    for (int e = 0; e < DH; e += 4) {
                        const float4 k = *(const float4 *)&s.k[j][e], v = *(const float4 *)&s.v[j][e];
                        const float4 q = *(const float4 *)&s.q[r][e], go = *(const float4 *)&s.dout[r][e];
                        x += q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
                        dp += go.x * v.x + go.y * v.y + go.z * v.z + go.w * v.w;
                    }
                }
                const bool vis = (sees >> j) & 1;
                const float p = vis ? exp2f(x * a.scale_log2 - l2) : 0.f;
                s.p[r][j] = p;
                s.ds[r][j] = vis ? p * (dp - delta) : 0.f;
            }
            __syncwarp();
            float dq[D];
#pragma unroll
            for (int d = 0; d < D; ++d) dq[d] = 0.f;
#pragma unroll 1
            for (uint64_t left = sees; left; left &= left - 1) {  // (what a row does not see may be NaN)
                const int j = __ffsll(left) - 1;
                const float w = s.ds[r][j];
#pragma unroll
                for (int d = 0; d < D; ++d) dq[d] += w * s.k[j][lane + 32 * d];
            }
            if (rr < a.R) {
#pragma unroll
                for (int d = 0; d < D; ++d) args.dq_new[(row0 + rr) * DH + lane + 32 * d] = dq[d];
            }
        }
        __syncthreads();
#pragma unroll 1
        for (int r = 0; r < ROWS; ++r) {
            const uint64_t sees = s.sees[r];
            if (!sees) continue;
            float q[D], go[D];
#pragma unroll
            for (int d = 0; d < D; ++d) q[d] = s.q[r][lane + 32 * d], go[d] = s.dout[r][lane + 32 * d];
#pragma unroll
            for (int j = 0; j < NW; ++j) {
                const int jj = j * WARPS + warp;  // (small trees: a node a warp)
                if (!((sees >> jj) & 1)) continue;
                const float w = s.ds[r][jj], p = s.p[r][jj];
#pragma unroll
                for (int d = 0; d < D; ++d) dk[j][d] += w * q[d], dv[j][d] += p * go[d];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < NW; ++j) {
        const int jj = j * WARPS + warp;
        if (jj >= a.N) continue;
        const size_t r = (size_t)b * a.N + jj;
#pragma unroll
        for (int d = 0; d < D; ++d) {
            store_elem(args.dk, a.dtype, r * a.ks + (size_t)g * DH + lane + 32 * d, dk[j][d] * args.scale);
            store_elem(args.dv, a.dtype, r * a.vs + (size_t)g * DH + lane + 32 * d, dv[j][d]);
        }
    }
}

// ---------------------------------------------------------------------------
// A block takes up to 32 / TW rows and a share of a sequence's cached tokens, four rows and 32 of TW times 32
// tokens a warp, so that few rows leave fewer warps idle; shares of a sequence for eight blocks an SM.  Bound by the
// latency of a tile's look-up, loads and products one after another: 40 sequences of 596 to 1988 tokens in 64-token
// pages, 8 kv heads of 128 fp32 dims: 4 rows 289 us (375 with TW = 1, 340 with longer shares), 32 rows 577 (654). The next
// tile's loads in registers beside the products take two of three blocks of an SM: 388 and 684.
template <int DH, int TW>
__global__ void __launch_bounds__(THREADS) tree_back_simt_kernel(const __grid_constant__ TreeBackArgs args) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    CacheSmem<DH, TW> &s = *(CacheSmem<DH, TW> *)smem_raw;
    const TreeArgs &a = args.t;
    constexpr int C = DH / 8, D = DH / 32, RWARPS = WARPS / TW, MINE = ROWS / TW, TILE = TOK * TW;
    pdl_wait();
    pdl_trigger();
    const int hv = blockIdx.y, g = hv / a.n_rb, rb = hv - g * a.n_rb, b = blockIdx.z, split = blockIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rw = warp % RWARPS, tg = warp / RWARPS;
    int *status = threadIdx.x == 0 && hv == 0 && split == 0 ? a.status : nullptr;
    const SeqRef sq = resolve_seq(a.seq_ids, a.seq_lens, 0, b, a.cache.kv.n_seqs, a.most_len, status);
    const int n = tree_nodes(a, b, nullptr);
    const int t_lo = (int)min((long long)sq.len, (long long)split * a.split_tokens);
    const int t_hi = t_lo + min(a.split_tokens, sq.len - t_lo);
    const int row0 = rb * a.rb_rows;
    for (int i = threadIdx.x; i < MINE * C; i += THREADS) {
        const int r = i / C, e = (i - r * C) * 8, rr = row0 + r;
        float q[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, go[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (rr < a.R && rr / a.G < n) {
            load_elems(a.q, a.dtype, row_at(a, b, g, rr, a.qs) + e, q);
            load_elems(args.dout, a.dtype, row_at(a, b, g, rr, (long long)a.Hq * DH) + e, go);
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) s.q[r][e + x] = q[x], s.dout[r][e + x] = go[x];
    }
    float dq[RW][D];
    float2 stat[RW];
#pragma unroll
    for (int r = 0; r < RW; ++r) {
        const int rr = row0 + rw * RW + r;
        stat[r] = rr < a.R ? args.stat[((size_t)b * a.Hkv + g) * a.R + rr] : make_float2(INFINITY, 0.f);
#pragma unroll
        for (int d = 0; d < D; ++d) dq[r][d] = 0.f;
    }
    const bool mine = row0 + rw * RW < a.R;  // (a warp without rows loads, and leaves shared memory to the others)
    bool bad = false;
    for (int t0 = t_lo; t0 < t_hi; t0 += TILE) {
        __syncthreads();
        for (int i = threadIdx.x; i < TILE * C; i += THREADS) {
            const int tt = i / C, e = (i - tt * C) * 8, t = t0 + tt;
            float k[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            long long row;
            int step;
            if (t < t_hi) {
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
            }
            store8(&s.k[tt][e], k);
            store8(&s.v[tt][e], v);
        }
        __syncthreads();
        const int here = min(TOK, t_hi - t0 - tg * TOK);
        if (!mine || here <= 0) continue;
        float x[RW] = {0.f, 0.f, 0.f, 0.f}, dp[RW] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int e = 0; e < DH; e += 4) {
            const float4 k = *(const float4 *)&s.k[tg * TOK + lane][e], v = *(const float4 *)&s.v[tg * TOK + lane][e];
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                const float4 q = *(const float4 *)&s.q[rw * RW + r][e], go = *(const float4 *)&s.dout[rw * RW + r][e];
                x[r] += q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
                dp[r] += go.x * v.x + go.y * v.y + go.z * v.z + go.w * v.w;
            }
        }
#pragma unroll
        for (int r = 0; r < RW; ++r) {
            const float p = lane < here ? exp2f(x[r] * a.scale_log2 - stat[r].x) : 0.f;
            x[r] = lane < here ? p * (dp[r] - stat[r].y) : 0.f;
        }
#pragma unroll 4
        for (int y = 0; y < here; ++y) {
            float kd[D];
#pragma unroll
            for (int d = 0; d < D; ++d) kd[d] = s.k[tg * TOK + y][lane + 32 * d];
#pragma unroll
            for (int r = 0; r < RW; ++r) {
                const float w = __shfl_sync(0xffffffffu, x[r], y);
#pragma unroll
                for (int d = 0; d < D; ++d) dq[r][d] += w * kd[d];
            }
        }
    }
    if (bad && a.status) atomicOr(a.status, SP_DEV_BAD_PAGE);
    const size_t slot = ((size_t)b * gridDim.y + hv) * a.n_splits + split;
    if constexpr (TW > 1) {  // the token groups' sums, added in their order
        float(*sum)[MINE][DH] = (float(*)[MINE][DH])smem_raw;
        static_assert(sizeof(float) * TW * MINE * DH <= sizeof s.k, "sums");
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RW; ++r)
#pragma unroll
            for (int d = 0; d < D; ++d) sum[tg][rw * RW + r][lane + 32 * d] = dq[r][d];
        __syncthreads();
        if (tg) return;
#pragma unroll
        for (int w = 1; w < TW; ++w)
#pragma unroll
            for (int r = 0; r < RW; ++r)
#pragma unroll
                for (int d = 0; d < D; ++d) dq[r][d] += sum[w][rw * RW + r][lane + 32 * d];
    }
#pragma unroll
    for (int r = 0; r < RW; ++r) {
        if (row0 + rw * RW + r >= a.R) continue;
#pragma unroll
        for (int d = 0; d < D; ++d) a.part_o[(slot * a.rb_rows + rw * RW + r) * DH + lane + 32 * d] = dq[r][d];
    }
}

// dq: the nodes' part and the shares' parts in share order, a warp a row, or (WIDE: many shares) a block a row
// whose warps take a run of shares each.
constexpr int MANY_SHARES = 16;
template <int DH, bool WIDE>
__global__ void __launch_bounds__(THREADS) tree_back_sum_kernel(const __grid_constant__ TreeBackArgs args) {
    const TreeArgs &a = args.t;
    constexpr int D = DH / 32;
    __shared__ float sums[WARPS][DH];
    pdl_wait();
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long w = WIDE ? blockIdx.x : (long long)blockIdx.x * WARPS + warp;
    if (w >= (long long)a.B * a.Hkv * a.R) return;
    const int rr = (int)(w % a.R), g = (int)(w / a.R % a.Hkv), b = (int)(w / a.R / a.Hkv);
    const int rb = rr / a.rb_rows;
    const size_t part0 = ((((size_t)b * a.Hkv + g) * a.n_rb + rb) * a.n_splits) * a.rb_rows + (rr - rb * a.rb_rows);
    const int per = WIDE ? ceil_div(a.n_splits, WARPS) : a.n_splits, lo = WIDE ? warp * per : 0, hi = min(a.n_splits, lo + per);
    float dq[D];
#pragma unroll
    for (int d = 0; d < D; ++d) dq[d] = !WIDE || warp == 0 ? args.dq_new[(size_t)w * DH + lane + 32 * d] : 0.f;
#pragma unroll 8
    for (int sp = lo; sp < hi; ++sp)
#pragma unroll
        for (int d = 0; d < D; ++d) dq[d] += a.part_o[(part0 + (size_t)sp * a.rb_rows) * DH + lane + 32 * d];
    if constexpr (WIDE) {
#pragma unroll
        for (int d = 0; d < D; ++d) sums[warp][lane + 32 * d] = dq[d];
        __syncthreads();
        if (warp) return;
#pragma unroll
        for (int i = 1; i < WARPS; ++i)
#pragma unroll
            for (int d = 0; d < D; ++d) dq[d] += sums[i][lane + 32 * d];
    }
    const bool live = args.stat[w].x != INFINITY;
#pragma unroll
    for (int d = 0; d < D; ++d)
        store_elem(args.dq, a.dtype, row_at(a, b, g, rr, a.qs) + lane + 32 * d, live ? dq[d] * args.scale : 0.f);
}

template <int DH>
cudaError_t run_rows(const TreeBackArgs &a, cudaStream_t st) {
    static bool known[MAX_DEVICES] = {};
    const cudaError_t e = allow_smem(tree_back_rows_kernel<DH>, (int)sizeof(RowSmem<DH>), known);
    if (e != cudaSuccess) return e;
    return launch_k(tree_back_rows_kernel<DH>, dim3(a.t.Hkv, a.t.B), dim3(THREADS), sizeof(RowSmem<DH>), st, a);
}
template <int DH, int TW>
cudaError_t run_cache(const TreeBackArgs &a, cudaStream_t st) {
    static bool known[MAX_DEVICES] = {};
    constexpr int bytes = (int)sizeof(CacheSmem<DH, TW>);
    const cudaError_t e = allow_smem(tree_back_simt_kernel<DH, TW>, bytes, known);
    if (e != cudaSuccess) return e;
    const TreeArgs &t = a.t;
    return launch_k(tree_back_simt_kernel<DH, TW>, dim3(t.n_splits, t.Hkv * t.n_rb, t.B), dim3(THREADS), (size_t)bytes, st, a);
}
template <int DH>
cudaError_t run_simt(const TreeBackArgs &a, cudaStream_t st) {
    const TreeArgs &t = a.t;
    const cudaError_t e = t.R <= ROWS / 2 ? run_cache<DH, 2>(a, st) : run_cache<DH, 1>(a, st);
    if (e != cudaSuccess) return e;
    const long long rows = (long long)t.B * t.Hkv * t.R;
    if (t.n_splits > MANY_SHARES) return launch_k(tree_back_sum_kernel<DH, true>, dim3((unsigned)rows), dim3(THREADS), 0, st, a);
    return launch_k(tree_back_sum_kernel<DH, false>, dim3((unsigned)ceil_div_ll(rows, WARPS)), dim3(THREADS), 0, st, a);
}

}  // namespace

size_t tree_back_simt_slots(const TreeArgs &a) { return (size_t)a.B * a.Hkv * a.n_rb * a.n_splits; }

cudaError_t launch_tree_back_simt(const TreeBackArgs &a, cudaStream_t st) {
    const cudaError_t e = a.t.dh == 128 ? run_rows<128>(a, st) : a.t.dh == 64 ? run_rows<64>(a, st) : run_rows<32>(a, st);
    if (e != cudaSuccess) return e;
    if (a.t.dh == 128) return run_simt<128>(a, st);
    if (a.t.dh == 64) return run_simt<64>(a, st);
    return run_simt<32>(a, st);
}

}  // namespace sp

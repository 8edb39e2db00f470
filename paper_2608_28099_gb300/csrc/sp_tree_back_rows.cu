// What of the backward pass of tree attention (sp_tree_back.cu) lies between the nodes, and the row
// statistics, for bf16 rows of 128 dims: a block a (sequence, kv head).  Five products of R rows, N
// nodes and 128 dims (scores, output gradients against values, dQ, dK, dV), too small for a tcgen05
// tile (64 x 16 at 16 soft-prompt rows and four heads a kv head): mma.sync on bf16 operands with fp32
// sums, a warp 16 rows, its weights' fragments going from the scores' accumulators into dQ's
// operand, dK and dV in registers over all rows, 128 / WARPS dims a warp.
//
// Operands enter the products finite: a non-finite element of a row or a node is taken out and
// remembered, and a weight (its gradient) between a row and a node that it sees becomes NaN where
// either of them has lost something that it needs.  So what a row does not see cannot reach it
// as 0 * NaN.
//
// For more than 16 nodes or several row blocks a kv head (sp_tree_back_tc.cu forms the others itself).
// Bound by latency: loads, two barriers and five short products a 64 rows; 32 sequences of 8 kv heads, 128
// rows and 32 nodes 11 us.
#include "sp_cache.cuh"
#include "sp_mma16.cuh"

namespace sp {

namespace {

constexpr int DH = 128, LD = DH + 8;  // elements of a row in shared memory (rows 4 banks apart)

template <int NP, int WARPS>
struct Smem {
    static constexpr int ROWS = 16 * WARPS;
    bf16 q[ROWS][LD], dout[ROWS][LD];
    bf16 k[NP][LD], v[NP][LD];
    bf16 p[ROWS][NP + 8], ds[ROWS][NP + 8];
    float2 stat[ROWS];                 // (log sum in log2 units, out.dout)
    unsigned long long sees[ROWS];
    unsigned odd_row[ROWS];            // bit 0: q, bit 1: dout held something not finite
    unsigned odd_node[NP];             // bit 0: k, bit 1: v
};

// NP: nodes, rounded up to 16, 32 or 64.
template <int NP, int WARPS>
__global__ void __launch_bounds__(32 * WARPS) tree_back_rows_tc_kernel(const __grid_constant__ TreeBackArgs args) {
    typedef Smem<NP, WARPS> Sm;
    constexpr int ROWS = Sm::ROWS;
    constexpr int MT = NP / 16, NT = DH / WARPS / 8;  // a warp's tiles of dK and dV: nodes, dims
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Sm &s = *(Sm *)smem_raw;
    const TreeArgs &a = args.t;
    pdl_wait();
    pdl_trigger();
    const int g = blockIdx.x, b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int c = lane & 15;  // 16 lanes a row: its 16-byte chunk
    const int n = tree_nodes(a, b, threadIdx.x == 0 && g == 0 ? a.status : nullptr);
    // nodes: a row of k and of v by 16 lanes each
    for (int j = warp * 2 + (lane >> 4); j < NP; j += WARPS * 2) {
        uint4 k = make_uint4(0, 0, 0, 0), v = k;
        if (j < n) {
            const size_t r = (size_t)b * a.N + j;
            k = *(const uint4 *)((const bf16 *)a.k_new + r * a.ks + (size_t)g * DH + c * 8);
            v = *(const uint4 *)((const bf16 *)a.v_new + r * a.vs + (size_t)g * DH + c * 8);
        }
        const unsigned half = 0xffffu << (lane & 16);
        const bool ko = __ballot_sync(0xffffffffu, take_finite(k)) & half, vo = __ballot_sync(0xffffffffu, take_finite(v)) & half;
        *(uint4 *)&s.k[j][c * 8] = k;
        *(uint4 *)&s.v[j][c * 8] = v;
        if (c == 0) s.odd_node[j] = (ko ? 1u : 0u) | (vo ? 2u : 0u);
    }
    float dk[MT][NT][4], dv[MT][NT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) dk[i][j][e] = dv[i][j][e] = 0.f;
    const size_t row0 = ((size_t)b * a.Hkv + g) * a.R;
#pragma unroll 1
    for (int r0 = 0; r0 < a.R; r0 += ROWS) {
        __syncthreads();  // (the rows before are read)
        // ---- 16 rows a warp: queries, output gradients, statistics; AT row pairs' loads under way together
        constexpr int AT = NP == 64 ? 2 : 4;
#pragma unroll 1
        for (int k0 = 0; k0 < 8; k0 += AT) {
            uint4 q[AT], go[AT], o[AT];
            float lse[AT];
            unsigned long long bits[AT];
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                const int rr = r0 + warp * 16 + (k0 + k) * 2 + (lane >> 4), node = rr / a.G;
                q[k] = go[k] = o[k] = make_uint4(0, 0, 0, 0);
                lse[k] = -INFINITY;
                bits[k] = 0;
                if (rr < a.R && node < n) {
                    const int head = g * a.G + rr - node * a.G;
                    const size_t row = (size_t)b * a.N + node, at = (row * a.Hq + head) * DH + c * 8;
                    q[k] = *(const uint4 *)((const bf16 *)a.q + row * a.qs + (size_t)head * DH + c * 8);
                    go[k] = *(const uint4 *)((const bf16 *)args.dout + at);
                    o[k] = *(const uint4 *)((const bf16 *)a.out + at);
                    lse[k] = a.lse[row * a.Hq + head];
                    bits[k] = tree_mask(a, b, node, n);
                }
            }
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                const int r = warp * 16 + (k0 + k) * 2 + (lane >> 4), rr = r0 + r;
                float d = dot8(go[k], o[k]);
#pragma unroll
                for (int x = 8; x; x >>= 1) d += __shfl_xor_sync(0xffffffffu, d, x);
                const unsigned half = 0xffffu << (lane & 16);
                const bool qo = __ballot_sync(0xffffffffu, take_finite(q[k])) & half;
                const bool oo = __ballot_sync(0xffffffffu, take_finite(go[k])) & half;
                *(uint4 *)&s.q[r][c * 8] = q[k];
                *(uint4 *)&s.dout[r][c * 8] = go[k];
                if (c == 0) {
                    float2 st = make_float2(INFINITY, 0.f);
                    if (lse[k] != -INFINITY) st = make_float2(lse[k] == INFINITY ? NAN : lse[k] * 1.4426950408889634f, d);
                    s.stat[r] = st;
                    s.sees[r] = st.x == INFINITY ? 0 : bits[k];
                    s.odd_row[r] = (qo ? 1u : 0u) | (oo ? 2u : 0u);
                    if (rr < a.R) args.stat[row0 + rr] = st;
                }
            }
        }
        __syncthreads();
        // ---- weights and their gradients of the warp's 16 rows
        const int wr = warp * 16, r_lo = wr + (lane >> 2), col = (lane & 3) * 2;
        uint32_t ds_frag[NP / 8][2];
        if (r0 + wr < a.R) {
            float x[NP / 8][4], dp[NP / 8][4];
#pragma unroll
            for (int j = 0; j < NP / 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[j][e] = dp[j][e] = 0.f;
#pragma unroll
            for (int kk = 0; kk < DH / 16; ++kk) {
                uint32_t qa[4], oa[4];
                ldsm4(qa, &s.q[wr + (lane & 15)][kk * 16 + (lane >> 4) * 8]);
                ldsm4(oa, &s.dout[wr + (lane & 15)][kk * 16 + (lane >> 4) * 8]);
#pragma unroll
                for (int j = 0; j < NP / 16; ++j) {  // 16 nodes: two operands of 8
                    uint32_t kb[4], vb[4];
                    const int node = j * 16 + (lane & 7) + (lane >> 4) * 8, d = kk * 16 + ((lane >> 3) & 1) * 8;
                    ldsm4(kb, &s.k[node][d]);
                    ldsm4(vb, &s.v[node][d]);
                    mma16816(x[2 * j], qa, kb[0], kb[1]);
                    mma16816(x[2 * j + 1], qa, kb[2], kb[3]);
                    mma16816(dp[2 * j], oa, vb[0], vb[1]);
                    mma16816(dp[2 * j + 1], oa, vb[2], vb[3]);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // rows r_lo and r_lo + 8
                const int r = r_lo + 8 * h;
                const float2 st = s.stat[r];
                const unsigned long long sees = s.sees[r];
                const unsigned odd = s.odd_row[r];
#pragma unroll
                for (int j = 0; j < NP / 8; ++j) {
                    float p[2], d[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int node = j * 8 + col + e;
                        const bool vis = (sees >> node) & 1;
                        const unsigned on = s.odd_node[node];
                        float w = fast_exp2(fmaf(x[j][2 * h + e], a.scale_log2, -st.x));
                        if ((odd | on) & 1u) w = NAN;
                        float z = w * (dp[j][2 * h + e] - st.y);
                        if ((odd | on) & 2u) z = NAN;
                        if (odd & 2u) w = NAN;
                        p[e] = vis ? w : 0.f;
                        d[e] = vis ? z : 0.f;
                    }
                    ds_frag[j][h] = pack2_bf16(d[0], d[1]);
                    *(uint32_t *)&s.p[r][j * 8 + col] = pack2_bf16(p[0], p[1]);
                    *(uint32_t *)&s.ds[r][j * 8 + col] = ds_frag[j][h];
                }
            }
            // ---- the nodes' part of dQ
#pragma unroll
            for (int d0 = 0; d0 < DH; d0 += 64) {
                float y[8][4];
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[j][e] = 0.f;
#pragma unroll
                for (int kk = 0; kk < NP / 16; ++kk) {
                    const uint32_t da[4] = {ds_frag[2 * kk][0], ds_frag[2 * kk][1], ds_frag[2 * kk + 1][0], ds_frag[2 * kk + 1][1]};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {  // 16 dims
                        uint32_t kb[4];
                        ldsm4t(kb, &s.k[kk * 16 + (lane & 15)][d0 + j * 16 + (lane >> 4) * 8]);
                        mma16816(y[2 * j], da, kb[0], kb[1]);
                        mma16816(y[2 * j + 1], da, kb[2], kb[3]);
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int rr = r0 + r_lo + 8 * h;
                    if (rr >= a.R) continue;
                    float *to = args.dq_new + (row0 + rr) * DH + d0 + col;
#pragma unroll
                    for (int j = 0; j < 8; ++j) *(float2 *)(to + j * 8) = make_float2(y[j][2 * h], y[j][2 * h + 1]);
                }
            }
        } else {  // rows that are not there: nothing to dK and dV
            for (int i = lane; i < 16 * NP / 2; i += 32) {
                const int r = wr + i / (NP / 2), x = i % (NP / 2) * 2;
                *(uint32_t *)&s.p[r][x] = 0;
                *(uint32_t *)&s.ds[r][x] = 0;
            }
        }
        __syncthreads();
        // ---- dK += ds^T Q, dV += p^T dO over the 16 WARPS rows, this warp's dims
        const int d0 = warp * (DH / WARPS);
#pragma unroll
        for (int kk = 0; kk < ROWS / 16; ++kk) {
            if (r0 + kk * 16 >= a.R) break;
            uint32_t qb[NT / 2][4], ob[NT / 2][4];
#pragma unroll
            for (int j = 0; j < NT / 2; ++j) {
                ldsm4t(qb[j], &s.q[kk * 16 + (lane & 15)][d0 + j * 16 + (lane >> 4) * 8]);
                ldsm4t(ob[j], &s.dout[kk * 16 + (lane & 15)][d0 + j * 16 + (lane >> 4) * 8]);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                // A = ds^T: nodes x rows, from rows x nodes
                uint32_t da[4], pa[4];
                const int r = kk * 16 + (lane & 7) + (lane >> 4) * 8, node = i * 16 + ((lane >> 3) & 1) * 8;
                ldsm4t(da, &s.ds[r][node]);
                ldsm4t(pa, &s.p[r][node]);
#pragma unroll
                for (int j = 0; j < NT / 2; ++j) {
                    mma16816(dk[i][2 * j], da, qb[j][0], qb[j][1]);
                    mma16816(dk[i][2 * j + 1], da, qb[j][2], qb[j][3]);
                    mma16816(dv[i][2 * j], pa, ob[j][0], ob[j][1]);
                    mma16816(dv[i][2 * j + 1], pa, ob[j][2], ob[j][3]);
                }
            }
        }
    }
    const int d0 = warp * (DH / WARPS) + (lane & 3) * 2;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int node = i * 16 + (lane >> 2) + 8 * h;
            if (node >= a.N) continue;
            const size_t r = (size_t)b * a.N + node;
            bf16 *tk = (bf16 *)args.dk + r * a.ks + (size_t)g * DH + d0, *tv = (bf16 *)args.dv + r * a.vs + (size_t)g * DH + d0;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                *(uint32_t *)(tk + j * 8) = pack2_bf16(dk[i][j][2 * h] * args.scale, dk[i][j][2 * h + 1] * args.scale);
                *(uint32_t *)(tv + j * 8) = pack2_bf16(dv[i][j][2 * h], dv[i][j][2 * h + 1]);
            }
        }
}

template <int NP, int WARPS>
cudaError_t run(const TreeBackArgs &a, cudaStream_t st) {
    static bool known[MAX_DEVICES] = {};
    constexpr int bytes = (int)sizeof(Smem<NP, WARPS>);
    const cudaError_t e = allow_smem(tree_back_rows_tc_kernel<NP, WARPS>, bytes, known);
    if (e != cudaSuccess) return e;
    return launch_k(tree_back_rows_tc_kernel<NP, WARPS>, dim3(a.t.Hkv, a.t.B), dim3(32 * WARPS), (size_t)bytes, st, a);
}

}  // namespace

cudaError_t launch_tree_back_rows_tc(const TreeBackArgs &a, cudaStream_t st) {
    if (a.t.N <= 16) return run<16, 4>(a, st);
    if (a.t.N <= 32) return run<32, 4>(a, st);
    return run<64, 8>(a, st);
}

}  // namespace sp

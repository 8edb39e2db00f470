// The cache's part of the backward pass of tree attention (sp_tree_back.cu) on tcgen05 tensor
// cores: head_dim 128, bf16 rows, bf16 or 8-bit cache.  Per key tile of 128 cached tokens and block of up to 128
// query rows of a kv head, rows on the MMA's M side:
//   S = Q K^T, dP = dO V^T   128 x 128 each, Q and dO in TMEM, K and V in shared memory
//   ds = p (dP - D)          p = exp(scale S - lse), a row a thread, written as bf16 over dP in TMEM
//   dQ += ds K               from TMEM; K is read a second time where it lies (MN-major)
// The log sums are known, so that a tile's weights are final: nothing is rescaled, two softmax
// warpgroups take half a tile's tokens each, and parts of dQ are sums.
//
// Work: the cached tokens of every sequence are cut into tiles, the list of all tiles into shares (as
// in sp_attn_plan.cuh), CTA (share, kv head, row block) walks its share; its piece of a sequence is
// a segment.  A pair that lies inside one share is finished there, the others leave partials that a second kernel adds in share order.
//
// Warps 0-7 softmax; 8-11 bring queries and output gradients (a segment ahead into shared memory,
// then into TMEM) and write dQ out; 12 MMA issuer and TMEM; 13 K, 14 V (TMA boxes of whole pages, cp.async
// elsewhere; 8-bit caches: 15 copies the codes, which 13 and 14 turn into bf16).  TMEM: S, dP, dQ, Q, dO in all 512 columns.  Every wait is time-limited
// (SP_DEV_TIMEOUT).
//
// What bounds it: HBM for long sequences.  Eight of 32768 tokens, 40 heads, 16 nodes (80 rows a kv head):
// 176 to 187 us, 5.8 to 6.1 TB/s; 64 of 1024 to 8192, 32 heads, 16 nodes: 210 to 233 us, 5.4 to 6.0 TB/s.  A tile's chain is
// dP (8 MMAs) -> ds -> dQ (8 MMAs), the next tile's S beside ds; an MMA with A in TMEM takes as long for 64
// tokens as for 128, which is why tiles have 128 tokens (64: 217 instead of 201 us for the eight, with two tiles
// under way), and Q and dO lie in TMEM (in shared memory 262 instead of 227, at 64 tokens).
// Short sequences are segment ends, 8 to 9 us of latencies one after another in warps 8-11 (200 sequences
// of 50 to 600 tokens: 111 us, 39 by bytes; 128 of 20 to 100: 50).  One sequence of 2048 tokens, 8 nodes: 14.6
// us, of which 5 are the second kernel and its launch.
// 8-bit caches: 355 us for the eight, 384 for 64 of 1024 to 8192 with 4 nodes (5980 and 1790 on CUDA cores), 3.3
// us a tile, no unit above 40 %: a tile's codes pass through one warp an operand (without their conversion
// 279 and 299, without the scales' products 336 and 370; two warps an operand, with 640 threads, 383 and 409;
// conversion by integer instructions 403 and 442).
// ds as a sum of two bf16 would halve its part of dQ's error (0.0031 -> 0.0025 of its norm) for 250 instead
// of 189 us.
#include <string.h>

#include "sp_attn_plan.cuh"
#include "sp_cache.cuh"
#include "sp_gemm.cuh"
#include "sp_mma16.cuh"

namespace sp {

namespace {

constexpr int TILE = 128;
constexpr int SLOT = TILE * DH * 2;             // K or V of a tile, 32 KB
constexpr int SCALES = 3 * TILE * 4;            // a tile's scales: of K times the scores' factor, of K, of V
constexpr int RAW = TILE * DH + 2 * TILE * 4;   // 8-bit codes of K or V, with K's the scales of both
constexpr int LD = DH + 8, STAGE_ROW = LD * 2;  // a staged row of queries or output gradients: elements, bytes
constexpr int MAX_NODES = 16;                   // most nodes whose products are formed here
constexpr int ROWS = 128;                       // most rows of a block
constexpr int MAX_RING = 8;
constexpr int BAR_EPI = 1;                      // named barrier of warps 8-11
constexpr int SMEM_MAX = 227 * 1024;
constexpr int THREADS = 512;
constexpr int EPI = 8, MMA = 12, K_WARP = 13, V_WARP = 14, COPY_WARP = 15;
constexpr uint32_t DP_COL = 128, DQ_COL = 256, Q_COL = 384, DO_COL = 448;  // TMEM: S, dP, dQ, Q, dO
// Fewest tiles a share holds on average (one sequence of 2048 tokens: 15.3, 14.7, 15.9 us with 1, 2, 3), and
// the cost of a segment in tiles (64 sequences of 1024 to 8192 tokens, 16 of 256 to 2048, 32 of 500 to 9000
// with 32 nodes: 234, 39, 182 us with 2; 226, 43, 188 with 8; 229, 44, 199 with 16).
constexpr int kBackMinTiles = 2;
constexpr int kBackSegCost = 5;

struct Layout {
    int nk, nv, nr;                             // ring slots of K and V, of 8-bit codes
    int off_q, off_do, off_n, off_ds, off_kn, off_k, off_v, off_sc, off_raw, off_tab;  // (off_q, off_do: staged rows; off_n:
                                                // Nodes; off_ds, off_kn: operands of the nodes' part of dQ;
                                                // 8-bit caches: off_sc: scales of the tiles in K's slots;
                                                // off_raw: codes of K or V of a tile, with K the scales of both)
    int smem;
};
struct Bars {
    uint64_t k_full[MAX_RING], k_empty[MAX_RING], v_full[MAX_RING], v_empty[MAX_RING];
    uint64_t s_full, s_read, d_full, p_full, n_full, q_full, q_empty, dq_full, dq_empty, fin;
    uint32_t tmem;
    int abort;
    int wsum[32];
    uint64_t raw_full[MAX_RING], raw_empty[MAX_RING];  // 8-bit caches
    int raw_meta[MAX_RING];
};
// What the segments' rows need, and the nodes of one.
struct Nodes {
    float2 stat[2][ROWS];              // by segment parity: (log sum in log2 units, out.dout)
    unsigned long long sees[ROWS];
    unsigned odd_row[ROWS];            // bit 0: q, bit 1: dout held something not finite
    unsigned odd_node[MAX_NODES];      // bit 0: k, bit 1: v
    bf16 v[MAX_NODES][LD];
};
constexpr int DS_BYTES = ROWS * MAX_NODES * 2;  // gradients of the weights between nodes: the A operand, 32-byte rows
constexpr int KN_BYTES = MAX_NODES * DH * 2;    // the nodes' keys: the B operand, by segment parity
constexpr int P_LD = MAX_NODES + 8;             // weights between nodes of 64 rows, in the other parity's place
static_assert(64 * P_LD * 2 <= KN_BYTES, "weights between nodes");
constexpr int OFF_CUTS = 1024;
constexpr int OFF_FRONT = OFF_CUTS + (MAX_GRP + 4) * 4;
static_assert(sizeof(Bars) <= OFF_CUTS, "barrier block");

__device__ __forceinline__ bool wait_warp(uint64_t *bar, uint32_t parity, volatile int *abort) {
    return mbar_wait_warp(bar, parity, abort);
}
__device__ __forceinline__ void arrive_warp(uint64_t *bar, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
}
__device__ __forceinline__ void expect_tx(uint64_t *bar, uint32_t bytes) {
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ld32_async(uint32_t addr, float *v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
          "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
          "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
          "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(addr));
}
// Earlier loads complete; these 32 values are named so that no use moves in front.
__device__ __forceinline__ void ld_wait(float *v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                   "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14])
                 :
                 : "memory");
    asm volatile(""
                 : "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]),
                   "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]));
    asm volatile("" : "+f"(v[29]), "+f"(v[30]), "+f"(v[31]));
}
__device__ __forceinline__ void st16_async(uint32_t addr, const uint32_t *v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The tile list: prefix[b] = tiles of the sequences before b (one for an empty sequence), each
// sequence's cache id, length and node count.  By all THREADS threads.
__device__ __forceinline__ void back_prefix(const TreeArgs &a, int *prefix, int *sids, int *lens, int *nodes, int *wsum,
                                            int *status, int *node_status) {
    const int B = a.B, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per = (B + THREADS - 1) / THREADS;
    const int b0 = min(B, (int)threadIdx.x * per), b1 = min(B, b0 + per);
    int sum = 0;
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
        const int n = a.n_nodes ? a.n_nodes[b] : a.N;  // (asked for beside the length)
        const SeqRef sq = resolve_seq(a.seq_ids, a.seq_lens, 0, b, a.cache.kv.n_seqs, a.most_len, status);
        sids[b] = sq.sid;
        lens[b] = sq.len;
        nodes[b] = checked_nodes(a, n, node_status);
        const int v = max(1, ceil_div(sq.len, TILE));
        prefix[b] = v;
        sum += v;
    }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) wsum[warp] = incl;
    __syncthreads();
    int run = incl - sum, tot = 0;
#pragma unroll 1
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) run += wsum[w];
        tot += wsum[w];
    }
#pragma unroll 1
    for (int b = b0; b < b1; ++b) {
        const int v = prefix[b];
        prefix[b] = run;
        run += v;
    }
    if (threadIdx.x == 0) prefix[B] = tot;
    __syncthreads();
}

struct Ring {
    int n, slot = 0;
    uint32_t ph = 0;
    __device__ __forceinline__ explicit Ring(int slots) : n(slots) {}
    __device__ __forceinline__ void next() {
        if (++slot == n) {
            slot = 0;
            ph ^= 1;
        }
    }
};
// A CTA's share: tiles [x0, x1) of the list, pieces of sequences [b0, b1).
struct Share {
    const int *prefix;
    int x0, x1, b0, b1;
};
__device__ __forceinline__ Seg piece(const Share &sh, int b) {
    const int p0 = sh.prefix[b], p1 = sh.prefix[b + 1], lo = max(p0, sh.x0);
    Seg s;
    s.b = b;
    s.xp = p0;
    s.nt = p1 - p0;
    s.t_a = lo - p0;
    s.n = min(p1, sh.x1) - lo;
    return s;
}
// Where a walk over the share's tiles stands: tile i of segment j (sequence b0 + j).
struct Walk {
    const Share &sh;
    Seg sg;
    int j = 0, i = 0;
    __device__ __forceinline__ explicit Walk(const Share &s) : sh(s) { sg = piece(sh, sh.b0); }
    __device__ __forceinline__ bool first() const { return i == 0; }
    __device__ __forceinline__ bool last() const { return i == sg.n - 1; }
    __device__ __forceinline__ void next() {
        if (++i < sg.n) return;
        i = 0;
        if (sh.b0 + ++j < sh.b1) sg = piece(sh, sh.b0 + j);
    }
};

// Queries and output gradients of sequence b, a block's rows, into their staging places; zeros for
// rows of nodes that are not there, and up to whole 16 rows.  16 lanes a row, four rows of each under
// way together.  NODES: the rows' statistics and what the products between nodes need of them, too.
template <bool NODES>
__device__ __forceinline__ void stage_rows(const TreeBackArgs &x, int b, int n, int g, int rb, uint8_t *Q, uint8_t *dO, Nodes *ns,
                                           float2 *stat, uint8_t *kn, bool owner, int wi, int lane) {
    const TreeArgs &a = x.t;
    const int c = lane & 15, rows = (a.rb_rows + 15) & ~15;
    constexpr int AT_ONCE = 4;
    uint4 nk[2], nv[2];  // the nodes' keys and values, under way beside the first rows
    if (NODES && owner) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = h * 8 + wi * 2 + (lane >> 4);
            nk[h] = nv[h] = make_uint4(0, 0, 0, 0);
            if (j < n) {
                const size_t r = (size_t)b * a.N + j;
                nk[h] = *(const uint4 *)((const bf16 *)a.k_new + r * a.ks + (size_t)g * DH + c * 8);
                nv[h] = *(const uint4 *)((const bf16 *)a.v_new + r * a.vs + (size_t)g * DH + c * 8);
            }
        }
    }
#pragma unroll 1
    for (int r1 = wi * 2 + (lane >> 4); r1 < rows; r1 += AT_ONCE * 8) {
        uint4 q[AT_ONCE], go[AT_ONCE], o[AT_ONCE];
        float lse[AT_ONCE];
        unsigned long long bits[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int r = r1 + k * 8, rr = rb * a.rb_rows + r, node = rr / a.G;
            q[k] = go[k] = o[k] = make_uint4(0, 0, 0, 0);
            lse[k] = -INFINITY;
            bits[k] = 0;
            if (r < a.rb_rows && rr < a.R && node < n) {
                const int hd = g * a.G + rr - node * a.G;
                const size_t head = (size_t)hd * DH + c * 8, row = (size_t)b * a.N + node;
                q[k] = *(const uint4 *)((const bf16 *)a.q + row * a.qs + head);
                go[k] = *(const uint4 *)((const bf16 *)x.dout + row * a.Hq * DH + head);
                if (NODES) {
                    o[k] = *(const uint4 *)((const bf16 *)a.out + row * a.Hq * DH + head);
                    lse[k] = a.lse[row * a.Hq + hd];
                    bits[k] = tree_mask(a, b, node, n);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int r = r1 + k * 8;  // (rows come in pairs: the warp's lanes agree on the end)
            if (r - (lane >> 4) >= rows) break;
            st_shared_v4(Q + r * STAGE_ROW + c * 16, q[k].x, q[k].y, q[k].z, q[k].w);
            st_shared_v4(dO + r * STAGE_ROW + c * 16, go[k].x, go[k].y, go[k].z, go[k].w);
            if constexpr (NODES) {
                float d = dot8(go[k], o[k]);
#pragma unroll
                for (int y = 8; y; y >>= 1) d += __shfl_xor_sync(0xffffffffu, d, y);
                const unsigned half = 0xffffu << (lane & 16);
                const bool qo = __ballot_sync(0xffffffffu, take_finite(q[k])) & half;
                const bool oo = __ballot_sync(0xffffffffu, take_finite(go[k])) & half;
                if (c == 0) {
                    float2 st = make_float2(INFINITY, 0.f);
                    if (lse[k] != -INFINITY) st = make_float2(lse[k] == INFINITY ? NAN : lse[k] * 1.4426950408889634f, d);
                    stat[r] = st;
                    ns->sees[r] = st.x == INFINITY ? 0 : bits[k];
                    ns->odd_row[r] = (qo ? 1u : 0u) | (oo ? 2u : 0u);
                }
            }
        }
    }
    if (NODES && owner) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = h * 8 + wi * 2 + (lane >> 4);
            const unsigned half = 0xffffu << (lane & 16);
            const bool ko = __ballot_sync(0xffffffffu, take_finite(nk[h])) & half;
            const bool vo = __ballot_sync(0xffffffffu, take_finite(nv[h])) & half;
            *(uint4 *)(kn + kv_off(j, c)) = nk[h];
            *(uint4 *)&ns->v[j][c * 8] = nv[h];
            if (c == 0) ns->odd_node[j] = (ko ? 1u : 0u) | (vo ? 2u : 0u);
        }
    }
}
// What lies between the nodes of sequence b (one row block, at most 16 nodes): gradients of their
// keys and values from the staged rows, and the A operand of their part of dQ, a last product of the
// segment's accumulator.  mma.sync by four warps that have nothing else to do while a segment's
// tiles are under way; the operands and what becomes of non-finite elements are those of
// sp_tree_back_rows.cu.
__device__ __forceinline__ void node_products(const TreeBackArgs &x, int b, int n, int g, uint8_t *Q, uint8_t *dO, Nodes &s,
                                              const float2 *stat, const uint8_t *kn, uint8_t *ds, bf16 *pw, int wi, int lane) {
    const TreeArgs &a = x.t;
    const int rows = (a.rb_rows + 15) & ~15;
    constexpr int NP = MAX_NODES, NT = DH / 4 / 8;
    {  // a row a thread: non-finite elements out (rare; the raw rows are in TMEM)
        const int r = wi * 32 + lane;
        if (r < rows && s.odd_row[r]) {
#pragma unroll 1
            for (int e = 0; e < DH * 2; e += 16) {
                uint4 q = *(uint4 *)(Q + r * STAGE_ROW + e), go = *(uint4 *)(dO + r * STAGE_ROW + e);
                take_finite(q);
                take_finite(go);
                *(uint4 *)(Q + r * STAGE_ROW + e) = q;
                *(uint4 *)(dO + r * STAGE_ROW + e) = go;
            }
        }
    }
    named_sync(BAR_EPI, 128);
    float dk[NT][4], dv[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) dk[j][e] = dv[j][e] = 0.f;
    const auto q_at = [&](int r, int d) { return (const bf16 *)(Q + r * STAGE_ROW) + d; };
    const auto o_at = [&](int r, int d) { return (const bf16 *)(dO + r * STAGE_ROW) + d; };
    const auto ds_at = [&](int r, int chunk) { return ds + r * 32 + ((chunk ^ (r >> 2 & 1)) << 4); };
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += 64) {
        if (r0) named_sync(BAR_EPI, 128);  // (the weights before are read)
        const int wr = wi * 16, r_lo = wr + (lane >> 2), col = (lane & 3) * 2;
        if (r0 + wr < rows) {
            float y[NP / 8][4], dp[NP / 8][4];
#pragma unroll
            for (int j = 0; j < NP / 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[j][e] = dp[j][e] = 0.f;
#pragma unroll
            for (int kk = 0; kk < DH / 16; ++kk) {
                uint32_t qa[4], oa[4], kb[4], vb[4];
                ldsm4(qa, q_at(r0 + wr + (lane & 15), kk * 16 + (lane >> 4) * 8));
                ldsm4(oa, o_at(r0 + wr + (lane & 15), kk * 16 + (lane >> 4) * 8));
                const int node = (lane & 7) + (lane >> 4) * 8, d = kk * 2 + ((lane >> 3) & 1);
                ldsm4(kb, kn + kv_off(node, d));
                ldsm4(vb, &s.v[node][d * 8]);
                mma16816(y[0], qa, kb[0], kb[1]);
                mma16816(y[1], qa, kb[2], kb[3]);
                mma16816(dp[0], oa, vb[0], vb[1]);
                mma16816(dp[1], oa, vb[2], vb[3]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int rl = r_lo + 8 * h, r = r0 + rl;
                const float2 st = stat[r];
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
                        float w = fast_exp2(fmaf(y[j][2 * h + e], a.scale_log2, -st.x));
                        if ((odd | on) & 1u) w = NAN;
                        float z = w * (dp[j][2 * h + e] - st.y);
                        if ((odd | on) & 2u) z = NAN;
                        if (odd & 2u) w = NAN;
                        p[e] = vis ? w : 0.f;
                        d[e] = vis ? z : 0.f;
                    }
                    *(uint32_t *)&pw[rl * P_LD + j * 8 + col] = pack_bf16(p[0], p[1]);
                    *(uint32_t *)(ds_at(r, j) + col * 2) = pack_bf16(d[0], d[1]);
                }
            }
        }
        named_sync(BAR_EPI, 128);
        const int d0 = wi * (DH / 4);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            if (r0 + kk * 16 >= rows) break;
            uint32_t da[4], pa[4];
            const int r = kk * 16 + (lane & 7) + (lane >> 4) * 8, chunk = (lane >> 3) & 1;
            ldsm4t(da, ds_at(r0 + r, chunk));
            ldsm4t(pa, &pw[r * P_LD + chunk * 8]);
#pragma unroll
            for (int j = 0; j < NT / 2; ++j) {
                uint32_t qb[4], ob[4];
                ldsm4t(qb, q_at(r0 + kk * 16 + (lane & 15), d0 + j * 16 + (lane >> 4) * 8));
                ldsm4t(ob, o_at(r0 + kk * 16 + (lane & 15), d0 + j * 16 + (lane >> 4) * 8));
                mma16816(dk[2 * j], da, qb[0], qb[1]);
                mma16816(dk[2 * j + 1], da, qb[2], qb[3]);
                mma16816(dv[2 * j], pa, ob[0], ob[1]);
                mma16816(dv[2 * j + 1], pa, ob[2], ob[3]);
            }
        }
    }
    const int d0 = wi * (DH / 4) + (lane & 3) * 2;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int node = (lane >> 2) + 8 * h;
        if (node >= a.N) continue;
        const size_t r = (size_t)b * a.N + node;
        bf16 *tk = (bf16 *)x.dk + r * a.ks + (size_t)g * DH + d0, *tv = (bf16 *)x.dv + r * a.vs + (size_t)g * DH + d0;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            *(uint32_t *)(tk + j * 8) = pack_bf16(dk[j][2 * h] * x.scale, dk[j][2 * h + 1] * x.scale);
            *(uint32_t *)(tv + j * 8) = pack_bf16(dv[j][2 * h], dv[j][2 * h + 1]);
        }
    }
}
// A staged row into 64 TMEM columns of its lane.
__device__ __forceinline__ void row_to_tmem(uint32_t addr, const uint8_t *row) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        uint32_t v[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 u = *(const uint4 *)(row + h * 64 + i * 16);
            v[4 * i] = u.x, v[4 * i + 1] = u.y, v[4 * i + 2] = u.z, v[4 * i + 3] = u.w;
        }
        st16_async(addr + h * 16, v);
    }
}

// 16 codes of row r (16-byte chunk c of its 128) as bf16, exactly, into a slot.
__device__ __forceinline__ void put_codes(uint8_t *slot, int r, int c, uint4 u) {
    const bool odd = c & 4;  // (the dim halves lie 1024 bytes apart: their lanes store chunks of other banks)
    const uint2 w[2] = {odd ? make_uint2(u.z, u.w) : make_uint2(u.x, u.y), odd ? make_uint2(u.x, u.y) : make_uint2(u.z, u.w)};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float v[8];
        codes_to_float(w[h], v);
        st_shared_v4(slot + kv_off(r, 2 * c + (h ? !odd : odd)), pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]),
                     pack_bf16(v[6], v[7]));
    }
}
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
        "l"(src), "r"(bytes), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void cp_async4(void *dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
// The 8-bit cache's codes and scales, copied by one warp (whole pages, or pieces of a row): K of a tile with
// the scales of both, V of it, and so on around one ring.
__device__ __forceinline__ void copy_codes(const TreeArgs &a, const Share &sh, const int *sids, const int *lens, int n_tiles, int g,
                                           Bars *bars, const Layout &lay, uint8_t *smem, volatile int *abort, int lane) {
    const bool paged = a.cache.kv.layout == SP_KV_PAGED;
    const int P = a.cache.kv.page_size, P_bits = 31 - __clz(max(P, 1)), Hkv = a.Hkv;
    struct Tile {
        int b, t0, n_tok, page;
    };
    int bad = 0;
    const auto ask = [&](const Walk &w) {  // (a lane's page)
        Tile t;
        t.b = sh.b0 + w.j;
        t.t0 = (w.sg.t_a + w.i) * TILE;
        t.n_tok = min(TILE, lens[t.b] - t.t0);
        t.page = -1;
        const int lp = (t.t0 >> P_bits) + lane;
        if (paged && lane * P < t.n_tok && lp < a.cache.kv.max_pages)
            t.page = __ldg(a.cache.kv.page_table + (size_t)sids[t.b] * a.cache.kv.max_pages + lp);
        return t;
    };
    Ring rg(lay.nr);
    int filled = 0;
    if (n_tiles > 0) {
        Walk at(sh);
        Tile t = ask(at);
#pragma unroll 1
        for (int x = 0; x < n_tiles; ++x) {
            Tile next = t;
            at.next();
            if (x + 1 < n_tiles) next = ask(at);
            const bool mine = paged && lane * P < t.n_tok, have = mine && t.page >= 0 && t.page < a.cache.kv.n_pages;
            if (mine && !have) bad = 1;
            const unsigned okm = __ballot_sync(0xffffffffu, have);
            // what the converting warps need: the groups of 16 rows that are there, and the tokens
            const int units = __ballot_sync(0xffffffffu, lane < 8 && lane * 16 < t.n_tok && (!paged || okm >> (lane * 16 >> P_bits) & 1));
            const int meta = units | max(t.n_tok, 0) << 8;
            const size_t row = paged ? ((size_t)t.page * Hkv + g) * P : (size_t)t.t0 * Hkv + g;  // (of a lane's page, if any)
#pragma unroll 1
            for (int is_v = 0; is_v < 2; ++is_v) {
                if (!wait_warp(&bars->raw_empty[rg.slot], rg.ph ^ 1, abort)) goto out;
                uint64_t *bar = &bars->raw_full[rg.slot];
                uint8_t *dst = smem + lay.off_raw + rg.slot * RAW;
                float *sc = (float *)(dst + TILE * DH);
                if (lane == 0) bars->raw_meta[rg.slot] = meta;
                if (mine && !have) {  // (scales behind the last token do not matter)
#pragma unroll 1
                    for (int r = lane * P; r < (lane + 1) * P; ++r) sc[r] = sc[TILE + r] = 0.f;
                }
                __syncwarp();
                // (a lane's stores are behind its own arrival where every lane arrives)
                if (!paged) mbar_arrive(bar);
                else if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)(__popc(okm) * P * (is_v ? DH : DH + 8)));
                __syncwarp();
                if (units) {
                    const uint8_t *src = (const uint8_t *)cache_base(a.cache, sids[t.b], is_v) + row * DH;
                    const float *k0 = is_v ? nullptr : scale_base(a.cache, sids[t.b], 0) + row;
                    const float *v0 = is_v ? nullptr : scale_base(a.cache, sids[t.b], 1) + row;
                    if (have) {
                        bulk_load(dst + lane * P * DH, src, P * DH, bar);
                        if (!is_v) {
                            bulk_load(sc + lane * P, k0, P * 4, bar);
                            bulk_load(sc + TILE + lane * P, v0, P * 4, bar);
                        }
                    } else if (!paged) {
                        const int r0 = lane >> 3, c = lane & 7;
                        const size_t step = (size_t)Hkv * DH;
                        src += r0 * step + c * 16;
#pragma unroll 4
                        for (int r = r0; r < t.n_tok; r += 4, src += 4 * step) cp_async16(dst + r * DH + c * 16, src);
                        if (!is_v) {
#pragma unroll 1
                            for (int r = lane; r < t.n_tok; r += 32) {
                                cp_async4(sc + r, k0 + (size_t)r * Hkv);
                                cp_async4(sc + TILE + r, v0 + (size_t)r * Hkv);
                            }
                        }
                    }
                }
                if (!paged) cp_async_mbar_arrive(bar);
                rg.next();
                ++filled;
            }
            t = next;
        }
    }
out:
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (lane == 0 && paged)  // copies still in flight (only possible after an abort): the last use of every slot
        for (int j = 1; j <= min(filled, rg.n); ++j)
            mbar_wait_drain(&bars->raw_full[(rg.slot - j + rg.n) % rg.n], rg.slot >= j ? rg.ph : rg.ph ^ 1);
    if (__any_sync(0xffffffffu, bad) && lane == 0 && a.status) atomicOr(a.status, SP_DEV_BAD_PAGE);
}
// Codes of K (or of V) to bf16 in that operand's ring, K's tiles with their scales.
__device__ __forceinline__ void convert_codes(bool is_v, float scale, int n_tiles, Bars *bars, const Layout &lay, uint8_t *smem, volatile int *abort,
                                              int lane) {
    const int r0 = lane >> 3, c = lane & 7;
    Ring rr(lay.nr), rg(is_v ? lay.nv : lay.nk);
    uint64_t *full = is_v ? bars->v_full : bars->k_full, *empty = is_v ? bars->v_empty : bars->k_empty;
    uint8_t *ring = smem + (is_v ? lay.off_v : lay.off_k);
    if (is_v) rr.next();
#pragma unroll 1
    for (int x = 0; x < n_tiles; ++x, rg.next(), rr.next(), rr.next()) {
        if (!wait_warp(&bars->raw_full[rr.slot], rr.ph, abort) || !wait_warp(&empty[rg.slot], rg.ph ^ 1, abort)) break;
        uint8_t *slot = ring + rg.slot * SLOT;
        const uint8_t *raw = smem + lay.off_raw + rr.slot * RAW;
        const int m = ((volatile int *)bars->raw_meta)[rr.slot], n_tok = m >> 8;
        if (!is_v) {
            const float4 *from = (const float4 *)(raw + TILE * DH);
            float4 *to = (float4 *)(smem + lay.off_sc + rg.slot * SCALES);
            const float4 k = from[lane];
            to[lane] = make_float4(k.x * scale, k.y * scale, k.z * scale, k.w * scale);
            to[32 + lane] = k;
            to[64 + lane] = from[32 + lane];
        }
        uint4 next[4];
        const auto load = [&](int i) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = i * 16 + k * 4 + r0;
                next[k] = make_uint4(0, 0, 0, 0);
                if ((m >> i & 1) && r < n_tok) next[k] = *(const uint4 *)(raw + r * DH + c * 16);
            }
        };
        load(0);
#pragma unroll 1
        for (int i = 0; i < TILE / 16; ++i) {
            uint4 now[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) now[k] = next[k];
            if (i + 1 < TILE / 16) load(i + 1);
#pragma unroll
            for (int k = 0; k < 4; ++k) put_codes(slot, i * 16 + k * 4 + r0, c, now[k]);
        }
        fence_proxy_async();
        mbar_arrive(&full[rg.slot]);
        arrive_warp(&bars->raw_empty[rr.slot], lane);
    }
}

// NODES: the row statistics and what lies between the nodes are formed here, else by a kernel in front.
// EIGHT: the cache holds 8-bit codes, whose scales enter S, dP and ds in fp32 (a bf16 holds a code, not its
// product with the scale).
template <bool NODES, bool EIGHT>
__global__ void __launch_bounds__(THREADS, 1)
    tree_back_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                        const __grid_constant__ TreeBackArgs args, const __grid_constant__ Layout lay, int2 *split_tab) {
    const TreeArgs &a = args.t;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Bars *bars = (Bars *)smem;
    int *cuts = (int *)(smem + OFF_CUTS);
    volatile int *abort = &bars->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int B = a.B, Hkv = a.Hkv, Hv = Hkv * a.n_rb;
    int *prefix = (int *)(smem + lay.off_tab), *sids = prefix + B + 1, *lens = sids + B, *nodes = lens + B;
    const bool paged = a.cache.kv.layout == SP_KV_PAGED;
    const int P = a.cache.kv.page_size, P_bits = 31 - __clz(max(P, 1));
    constexpr int ROW = DH * 2;
    // The first kernel of its call reads nothing of the caller's before the wait.  Behind a kernel of the
    // call, which has waited before it let this one start: lengths, counts, queries and the cache may be
    // read, that kernel's results only behind the wait.
    if (NODES) pdl_wait();
    Nodes *ns = (Nodes *)(smem + lay.off_n);
    back_prefix(a, prefix, sids, lens, nodes, bars->wsum, blockIdx.x == 0 ? a.status : nullptr,
                NODES && blockIdx.x == 0 ? a.status : nullptr);
    const int T = prefix[B];
    const int n_grp = share_count((int)gridDim.x / Hv, T, B, a.plan.tc_min_tiles);
    const int grp = blockIdx.x / Hv, hv = blockIdx.x - grp * Hv, g = hv / a.n_rb, rb = hv - g * a.n_rb;
    if (grp >= n_grp) return;  // uniform over the CTA: no share
    if (threadIdx.x < PLAN_THREADS) build_cuts(a.plan, prefix, T, n_grp, cuts, bars->wsum);
    if (threadIdx.x == THREADS - 1) {
#pragma unroll 1
        for (int i = 0; i < lay.nk; ++i) {
            mbar_init(&bars->k_full[i], 32);
            mbar_init(&bars->k_empty[i], 1);
        }
#pragma unroll 1
        for (int i = 0; i < lay.nv; ++i) {
            mbar_init(&bars->v_full[i], 32);
            mbar_init(&bars->v_empty[i], 1);
        }
        if (EIGHT) {
#pragma unroll 1
            for (int i = 0; i < lay.nr; ++i) {
                mbar_init(&bars->raw_full[i], paged ? 1 : 64);
                mbar_init(&bars->raw_empty[i], 1);
            }
        }
        mbar_init(&bars->s_full, 1);
        mbar_init(&bars->s_read, 8);
        mbar_init(&bars->d_full, 1);
        mbar_init(&bars->p_full, 8);
        mbar_init(&bars->n_full, 4);
        mbar_init(&bars->q_full, 4);
        mbar_init(&bars->q_empty, 1);
        mbar_init(&bars->dq_full, 1);
        mbar_init(&bars->dq_empty, 4);
        mbar_init(&bars->fin, 1);
        bars->abort = 0;
        fence_mbar_init();
        if (paged && !EIGHT) {
            prefetch_tmap(&map_k);
            prefetch_tmap(&map_v);
        }
    }
    if (warp == MMA) {
        tmem_alloc(&bars->tmem, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars->tmem;
    Share sh{prefix, cuts[grp], cuts[grp + 1], 0, 0};
    if (sh.x0 < sh.x1) {
        sh.b0 = seg_at(prefix, B, sh.x0, sh.x1).b;
        sh.b1 = seg_at(prefix, B, sh.x1 - 1, sh.x1).b + 1;
    }
    const int n_tiles = max(sh.x1 - sh.x0, 0);
    if (blockIdx.x == 0) {  // for the merge: the sequence that goes on behind the share where it starts, its shares
#pragma unroll 1
        for (int j = threadIdx.x; j < (int)gridDim.x / Hv; j += THREADS) {
            int2 t = make_int2(0, 0);
            if (j < n_grp && cuts[j] < cuts[j + 1]) {
                const int b = seg_at(prefix, B, cuts[j + 1] - 1, T).b;
                if (prefix[b] >= cuts[j]) t = make_int2(b, group_of(cuts, n_grp, prefix[b + 1] - 1) - j + 1);
            }
            split_tab[j] = t;
        }
    }

    if (warp < 8) {
        // ------------------------------------------------------------ weights and their gradients
        const int c0 = (warp >> 2) * 64, r = threadIdx.x & 127;  // this warpgroup's tokens of a tile; row, TMEM lane
        const int rr = rb * a.rb_rows + r;
        const bool active = r < a.rb_rows && rr < a.R;
        const bool warp_active = __any_sync(0xffffffffu, active);
        const uint32_t s_col = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)c0;
        if (!NODES) pdl_wait();  // the row statistics
        bool ok = true;
        uint32_t ph = 0;
        Ring rs(lay.nk);
#pragma unroll 1
        for (int b = sh.b0; ok && b < sh.b1; ++b) {
            const Seg sg = piece(sh, b);
            const int left = lens[b] - sg.t_a * TILE - c0;
            float2 st = make_float2(INFINITY, 0.f);
            if (!NODES && active) st = __ldcg(args.stat + ((size_t)b * Hkv + g) * a.R + rr);
#pragma unroll 1
            for (int i = 0; i < sg.n; ++i, ph ^= 1, rs.next()) {
                ok = ok && wait_warp(&bars->s_full, ph, abort);
                if (!ok) break;
                tc_fence_after();
                // (there since the queries are: the scores waited for both)
                if (NODES && i == 0 && active) {
                    const volatile float *at = &ns->stat[(b - sh.b0) & 1][r].x;
                    st = make_float2(at[0], at[1]);
                }
                // the tile's scales, there with its keys, which stay until its dQ is formed
                const float4 *kf = (const float4 *)(smem + lay.off_sc + rs.slot * SCALES + c0 * 4), *ks = kf + TILE / 4, *vs = ks + TILE / 4;
                if (EIGHT) ok = wait_warp(&bars->k_full[rs.slot], rs.ph, abort);
                if (!ok) break;
                const int n_tok = left - i * TILE;
                float s[64];
                if (warp_active) {  // the weights, while dP is formed
                    ld32_async(s_col, s);
                    ld32_async(s_col + 32, s + 32);
                    ld_wait(s);
                    ld_wait(s + 32);
                    if constexpr (EIGHT) {
#pragma unroll
                        for (int e = 0; e < 64; e += 4) {
                            const float4 f = kf[e / 4];
                            s[e] = fast_exp2(fmaf(s[e], f.x, -st.x)), s[e + 1] = fast_exp2(fmaf(s[e + 1], f.y, -st.x));
                            s[e + 2] = fast_exp2(fmaf(s[e + 2], f.z, -st.x)), s[e + 3] = fast_exp2(fmaf(s[e + 3], f.w, -st.x));
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 64; ++e) s[e] = fast_exp2(fmaf(s[e], a.scale_log2, -st.x));
                    }
                    tc_fence_before();
                }
                arrive_warp(&bars->s_read, lane);  // the next scores may be formed
                ok = wait_warp(&bars->d_full, ph, abort);
                if (!ok) break;
                tc_fence_after();
                if (warp_active) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float d[32];
                        ld32_async(s_col + DP_COL + c * 32, d);
                        ld_wait(d);
                        if constexpr (EIGHT) {
#pragma unroll
                            for (int e = 0; e < 32; e += 4) {
                                const float4 f = vs[c * 8 + e / 4], k = ks[c * 8 + e / 4];
                                d[e] *= f.x, d[e + 1] *= f.y, d[e + 2] *= f.z, d[e + 3] *= f.w;
                                s[c * 32 + e] *= k.x, s[c * 32 + e + 1] *= k.y, s[c * 32 + e + 2] *= k.z, s[c * 32 + e + 3] *= k.w;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 32; ++e) d[e] = s[c * 32 + e] * (d[e] - st.y);
                        if (n_tok < c * 32 + 32) {  // past the end: what was loaded there is nothing
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (c * 32 + e >= n_tok) d[e] = 0.f;
                        }
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) pk[e] = pack_bf16(d[2 * e], d[2 * e + 1]);
                        st16_async(s_col + DP_COL + c * 16, pk);  // over products that this warp has read
                    }
                    st_wait();
                }
                tc_fence_before();
                arrive_warp(&bars->p_full, lane);
            }
        }
    } else if (warp < MMA) {
        // ------------------------------------------------------------ queries in, dQ out
        const int quad = warp - EPI, r = quad * 32 + lane, rr = rb * a.rb_rows + r;
        const bool active = r < a.rb_rows && rr < a.R;
        const bool warp_active = __any_sync(0xffffffffu, active);
        const uint32_t lane_base = tmem + ((uint32_t)(quad * 32) << 16);
        const int n_seg = sh.b1 - sh.b0;
        // the rows of segment j: staged; into TMEM once the scores before have read theirs
        const auto load = [&](int j) {
            const int b = sh.b0 + j;
            named_sync(BAR_EPI, 128);  // (the staged rows before are in TMEM)
            stage_rows<NODES>(args, b, nodes[b], g, rb, smem + lay.off_q, smem + lay.off_do, ns, ns->stat[j & 1],
                              smem + lay.off_kn + (j & 1) * KN_BYTES, sh.x0 <= prefix[b], quad, lane);
            named_sync(BAR_EPI, 128);
            const bool free = wait_warp(&bars->q_empty, (j & 1) ^ 1, abort);
            if (free && warp_active) {
                tc_fence_after();
                const int from = min(r, a.rb_rows - 1);  // (lanes behind the rows: any)
                row_to_tmem(lane_base + Q_COL, smem + lay.off_q + from * STAGE_ROW);
                row_to_tmem(lane_base + DO_COL, smem + lay.off_do + from * STAGE_ROW);
                st_wait();
                tc_fence_before();
            }
            if (free) arrive_warp(&bars->q_full, lane);
            return free;
        };
        // (a warp whose wait ran out goes on to the barriers that the others meet at)
        bool ok = n_seg == 0 || load(0);
        if (!NODES) pdl_wait();  // the nodes' part of dQ; nothing is written before
        // the share that has a sequence's first tile forms what lies between its nodes
        const auto between = [&](int j) {
            const int b = sh.b0 + j;
            if (!NODES || sh.x0 > prefix[b]) return;
            const float2 *stat = ns->stat[j & 1];
            node_products(args, b, nodes[b], g, smem + lay.off_q, smem + lay.off_do, *ns, stat, smem + lay.off_kn + (j & 1) * KN_BYTES,
                          smem + lay.off_ds, (bf16 *)(smem + lay.off_kn + (~j & 1) * KN_BYTES), quad, lane);
            if (active) args.stat[((size_t)b * Hkv + g) * a.R + rr] = stat[r];
            fence_proxy_async();  // ds and the nodes' keys -> tensor-core reads
            arrive_warp(&bars->n_full, lane);
        };
        if (n_seg > 0) between(0);
#pragma unroll 1
        for (int j = 0; j < n_seg; ++j) {
            if (j + 1 < n_seg) ok = load(j + 1) && ok;
            const int b = sh.b0 + j;
            const Seg sg = piece(sh, b);
            const int n = nodes[b];
            // slot of a partial: a share has at most two, of the pair that starts in it and of the one that began before
            const bool starts = sg.xp >= sh.x0, whole = starts && sg.xp + sg.nt <= sh.x1;
            const size_t slot = ((size_t)grp * 2 + starts) * Hv + hv;
            const int node = rr / a.G;
            const size_t row = ((size_t)b * Hkv + g) * a.R + rr;
            bool live = false;
            if (active && whole) live = node < n && (NODES ? ns->stat[j & 1][r].x : __ldcg(&args.stat[row].x)) != INFINITY;
            ok = ok && wait_warp(&bars->dq_full, j & 1, abort);
            if (ok && warp_active) {
                tc_fence_after();
                float *part = a.part_o + (slot * a.rb_rows + r) * DH;
                bf16 *to = (bf16 *)args.dq + ((size_t)b * a.N + node) * a.qs + (size_t)(g * a.G + rr - node * a.G) * DH;
                const float4 *more = (const float4 *)(args.dq_new + row * DH);
                const float f = args.scale;
#pragma unroll 1
                for (int d = 0; d < DH; d += 32) {
                    float v[32];
                    __syncwarp();
                    ld32_async(lane_base + DQ_COL + (uint32_t)d, v);
                    ld_wait(v);
                    if (!active) continue;
                    if (whole) {
                        if (!NODES) {
#pragma unroll
                            for (int e = 0; e < 32; e += 4) {
                                const float4 y = __ldcg(more + (d + e) / 4);
                                v[e] += y.x, v[e + 1] += y.y, v[e + 2] += y.z, v[e + 3] += y.w;
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 32; e += 8)
                            *(uint4 *)(to + d + e) = live ? make_uint4(pack_bf16(v[e] * f, v[e + 1] * f), pack_bf16(v[e + 2] * f, v[e + 3] * f),
                                                                       pack_bf16(v[e + 4] * f, v[e + 5] * f), pack_bf16(v[e + 6] * f, v[e + 7] * f))
                                                          : make_uint4(0, 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) *(float4 *)(part + d + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                    }
                }
                tc_fence_before();
            }
            if (ok) arrive_warp(&bars->dq_empty, lane);
            if (j + 1 < n_seg) between(j + 1);
        }
    } else if (EIGHT && warp >= K_WARP) {
        if (warp == COPY_WARP) copy_codes(a, sh, sids, lens, n_tiles, g, bars, lay, smem, abort, lane);
        else convert_codes(warp == V_WARP, a.scale_log2, n_tiles, bars, lay, smem, abort, lane);
    } else if (!EIGHT && (warp == K_WARP || warp == V_WARP)) {
        // ------------------------------------------------------------ K and V
        const bool is_v = warp == V_WARP;
        uint64_t *full = is_v ? bars->v_full : bars->k_full, *empty = is_v ? bars->v_empty : bars->k_empty;
        uint8_t *ring = smem + (is_v ? lay.off_v : lay.off_k);
        const CUtensorMap *map = is_v ? &map_v : &map_k;
        const uint8_t *pool = (const uint8_t *)(is_v ? a.cache.kv.v_pool : a.cache.kv.k_pool);
        const uint64_t pol = policy_evict_first();
        Ring rg(is_v ? lay.nv : lay.nk);
        int bad = 0, filled = 0;
        // the tile's page ids, a lane each (-1: none), asked for a tile ahead: an answer that comes behind
        // the cache stream takes longer than a tile
        const auto ask = [&](const Walk &w) {
            const int b = sh.b0 + w.j, t0 = (w.sg.t_a + w.i) * TILE, lp = (t0 >> P_bits) + lane;
            if (!paged || lane * P >= min(TILE, lens[b] - t0) || lp >= a.cache.kv.max_pages) return -1;
            return __ldg(a.cache.kv.page_table + (size_t)sids[b] * a.cache.kv.max_pages + lp);
        };
        if (n_tiles > 0) {
            Walk at(sh);
            int next = ask(at);
#pragma unroll 1
            for (int x = 0; x < n_tiles; ++x) {
                const int b = sh.b0 + at.j, t0 = (at.sg.t_a + at.i) * TILE, n_tok = min(TILE, lens[b] - t0);
                const int n_pg = paged ? n_tok >> P_bits : 0;  // whole pages
                int page = next;
                if (paged && lane * P < n_tok && (page < 0 || page >= a.cache.kv.n_pages)) page = -1, bad = 1;
                at.next();
                if (x + 1 < n_tiles) next = ask(at);
                // warp-uniform verdict: the collectives below need every lane
                if (!wait_warp(&empty[rg.slot], rg.ph ^ 1, abort)) break;
                uint8_t *dst = ring + rg.slot * SLOT;
                bool plain = false;  // this thread wrote shared memory or issued cp.async
                if (n_pg > 0) {
                    const bool have = lane < n_pg && page >= 0;
                    const unsigned okm = __ballot_sync(0xffffffffu, have);
                    if (lane == 0 && okm) expect_tx(&full[rg.slot], __popc(okm) * P * ROW);
                    __syncwarp();
                    if (have)  // the cache is read once: evict-first keeps queries and partials in L2
                        tma_load_4d_hint(dst + lane * P * ROW, map, &full[rg.slot], 0, 0, 0, (page * Hkv + g) * (P / 8), pol);
#pragma unroll 1
                    for (unsigned miss = ~okm & ((1u << n_pg) - 1u); miss; miss &= miss - 1) {  // zeros
                        const int j = __ffs(miss) - 1;
#pragma unroll 1
                        for (int e = lane; e < P * ROW / 16; e += 32) st_shared_v4(dst + j * P * ROW + e * 16, 0, 0, 0, 0);
                        plain = true;
                    }
                }
                const int r0 = n_pg * (paged ? P : 0);  // first row not covered by TMA
                if (r0 < n_tok) {
                    plain = true;
                    const uint8_t *src;
                    size_t step = ROW;
                    bool have = true;
                    if (!paged) {  // a contiguous sequence's rows of head g, a token apart
                        step = (size_t)Hkv * ROW;
                        src = (const uint8_t *)(is_v ? a.cache.kv.v_seq : a.cache.kv.k_seq)[sids[b]] + (size_t)g * ROW + (size_t)t0 * step;
                    } else {  // the last, partial page
                        const int pg = __shfl_sync(0xffffffffu, page, n_pg);
                        have = pg >= 0;
                        src = pool + ((size_t)max(pg, 0) * Hkv + g) * P * ROW;
                    }
                    const int c = lane & 15, r1 = lane >> 4;
                    src += (size_t)r1 * step + c * 16;
#pragma unroll 4
                    for (int r = r1; r < n_tok - r0; r += 2, src += 2 * step) {
                        uint8_t *d = dst + kv_off(r0 + r, c);
                        if (have) cp_async16(d, src);
                        else st_shared_v4(d, 0, 0, 0, 0);
                    }
                }
                if (n_tok < TILE) {  // rows past the end meet gradients of 0: they must be finite
                    plain = true;
                    const int from = max(n_tok, 0);
#pragma unroll 1
                    for (int idx = lane; idx < (TILE - from) * 16; idx += 32)
                        st_shared_v4(dst + kv_off(from + (idx >> 4), idx & 15), 0, 0, 0, 0);
                }
                if (plain) {
                    fence_proxy_async();  // this thread's shared-memory stores
                    cp_async_mbar_arrive(&full[rg.slot]);
                } else {
                    mbar_arrive(&full[rg.slot]);
                }
                ++filled;
                rg.next();
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");  // nothing lands after the CTA is gone
        if (lane == 0)  // bulk copies still in flight (only possible after an abort): the last use of every slot
            for (int j = 0; j < min(filled, rg.n); ++j) {
                const int back = j + 1, slot = (rg.slot - back + rg.n) % rg.n;
                mbar_wait_drain(&full[slot], rg.slot >= back ? rg.ph : rg.ph ^ 1);
            }
        bad = __any_sync(0xffffffffu, bad);
        if (bad && lane == 0 && a.status) atomicOr(a.status, SP_DEV_BAD_PAGE);
    } else if (warp == MMA) {
        // ------------------------------------------------------------ MMA issue
        // One issuer.  Per tile x: dP, beside which the softmax forms the weights; the scores of tile
        // x + 1 as soon as it has read those of x, beside which it forms ds (over dP); dQ, which is in front
        // of the next dP in the pipe.  Where tile x + 1 begins a segment whose queries are not there
        // yet, its scores come behind dQ.
        const bool on = elect_one();
        constexpr uint32_t idesc_s = idesc_bf16_f32(128, TILE), idesc_q = idesc_bf16_f32_bmn(128, DH);
        const uint64_t dk0 = sw128_kmajor_desc_sbo(smem + lay.off_k, GROUP_STRIDE);
        const uint64_t dv0 = sw128_kmajor_desc_sbo(smem + lay.off_v, GROUP_STRIDE);
        const uint64_t dkt0 = sw128_mnmajor_desc2(smem + lay.off_k, HALF_STRIDE, GROUP_STRIDE);
        Ring rk(lay.nk), rv(lay.nv), rk2(lay.nk);  // of S, of dP, of dQ
        bool ok = n_tiles > 0;
        if (ok) {
            Walk in(sh), at(sh);                   // the tiles of S, of dP and dQ
            int scored = 0;
            uint32_t n_ph = 0;
            const auto scores = [&]() {
                if (in.first()) ok = wait_warp(&bars->q_full, in.j & 1, abort);
                ok = ok && wait_warp(&bars->k_full[rk.slot], rk.ph, abort);
                if (scored > 0) ok = ok && wait_warp(&bars->s_read, (scored - 1) & 1, abort);
                if (!ok) return;
                tc_fence_after();
                fence_proxy_async();  // cp.async data -> tensor-core reads
                const uint64_t k = dk0 + (uint32_t)(rk.slot * (SLOT >> 4));
                if (on) {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)  // 16 dims: 8 columns of Q, 32 B of a row of K's dim half kk / 4
                        mma_bf16_ts(tmem, tmem + Q_COL + (uint32_t)(kk * 8),
                                    k + (uint64_t)((kk >> 2) * (HALF_STRIDE >> 4) + (kk & 3) * 2), idesc_s, kk > 0);
                    mma_commit(&bars->s_full);
                }
                __syncwarp();
                rk.next();
                in.next();
                ++scored;
            };
            scores();
#pragma unroll 1
            for (int x = 0; ok && x < n_tiles; ++x) {
                ok = wait_warp(&bars->v_full[rv.slot], rv.ph, abort);
                if (!ok) break;
                tc_fence_after();
                fence_proxy_async();
                const uint64_t v = dv0 + (uint32_t)(rv.slot * (SLOT >> 4));
                if (on) {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        mma_bf16_ts(tmem + DP_COL, tmem + DO_COL + (uint32_t)(kk * 8),
                                    v + (uint64_t)((kk >> 2) * (HALF_STRIDE >> 4) + (kk & 3) * 2), idesc_s, kk > 0);
                    mma_commit(&bars->d_full);
                    mma_commit(&bars->v_empty[rv.slot]);
                    if (at.last()) mma_commit(&bars->q_empty);
                }
                __syncwarp();
                if (x + 1 < n_tiles && (!in.first() || __all_sync(0xffffffffu, mbar_try_wait(&bars->q_full, in.j & 1)))) scores();
                // (the segment before: its dQ has been read)
                if (at.first() && at.j >= 1) ok = ok && wait_warp(&bars->dq_empty, (at.j - 1) & 1, abort);
                ok = ok && wait_warp(&bars->p_full, x & 1, abort);
                if (!ok) break;
                tc_fence_after();
                const uint64_t kt = dkt0 + (uint32_t)(rk2.slot * (SLOT >> 4));
                if (on) {
#pragma unroll
                    for (int kk = 0; kk < TILE / 16; ++kk)  // 16 tokens: 8 columns of ds (of its half's), two 8-token groups of K
                        mma_bf16_ts(tmem + DQ_COL, tmem + DP_COL + (uint32_t)((kk >> 2) * 64 + (kk & 3) * 8),
                                    kt + (uint64_t)(kk * (2 * GROUP_STRIDE >> 4)), idesc_q, kk > 0 || !at.first());
                    mma_commit(&bars->k_empty[rk2.slot]);
                }
                __syncwarp();
                if (at.last()) {
                    const bool mine = NODES && sh.x0 <= prefix[sh.b0 + at.j];  // the nodes' part, by their sequence's first share
                    if (mine) {
                        ok = wait_warp(&bars->n_full, n_ph, abort);
                        n_ph ^= 1;
                        if (!ok) break;
                        tc_fence_after();
                        fence_proxy_async();
                    }
                    if (on) {
                        if (mine)
                            mma_bf16(tmem + DQ_COL, sw32_kmajor_desc(smem + lay.off_ds),
                                     sw128_mnmajor_desc2(smem + lay.off_kn + (at.j & 1) * KN_BYTES, HALF_STRIDE, GROUP_STRIDE), idesc_q, 1u);
                        mma_commit(&bars->dq_full);
                    }
                    __syncwarp();
                }
                rk2.next();
                rv.next();
                at.next();
                if (x + 1 < n_tiles && scored == x + 1) scores();
            }
        }
        if (on) mma_commit(&bars->fin);  // completes when every MMA is done
        __syncwarp();
    }
    // every MMA must be finished before TMEM and shared memory go away
    mbar_wait_drain(&bars->fin, 0);
    tc_fence_before();
    __syncthreads();
    pdl_trigger();
    if (threadIdx.x == 0 && *abort && a.status) atomicOr(a.status, SP_DEV_TIMEOUT);
    if (warp == MMA) tmem_dealloc(tmem, 512);
}

// dQ of the pairs that lie in several shares (at most one starts in each share): a warp per (share,
// kv head, row), four dims a lane, the partials in share order, SUM_AT of them under way together.
constexpr int SUM_THREADS = 128, SUM_ROWS = SUM_THREADS / 32, SUM_AT = 8;
__global__ void __launch_bounds__(SUM_THREADS) tree_back_tc_sum_kernel(const __grid_constant__ TreeBackArgs args, const int2 *split_tab, int add_nodes) {
    const TreeArgs &a = args.t;
    pdl_wait();
    const int hv = blockIdx.x, j0 = blockIdx.y, Hv = a.Hkv * a.n_rb, g = hv / a.n_rb, rb = hv - g * a.n_rb;
    const int2 tab = __ldcg(split_tab + j0);
    if (tab.y <= 1) return;
    const int b = tab.x, lane = threadIdx.x & 31, c = lane * 4;
    const int q = blockIdx.z * SUM_ROWS + (threadIdx.x >> 5), rr = rb * a.rb_rows + q;
    if (q >= a.rb_rows || rr >= a.R) return;
    const size_t at = ((size_t)b * a.Hkv + g) * a.R + rr;
    float4 s = add_nodes ? __ldcg((const float4 *)(args.dq_new + at * DH + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
    const bool live = __ldcg(&args.stat[at].x) != INFINITY;  // (+inf for a node that is not there, too)
#pragma unroll 1
    for (int e0 = 0; e0 < tab.y; e0 += SUM_AT) {
        float4 v[SUM_AT];
#pragma unroll
        for (int e = 0; e < SUM_AT; ++e) {
            const size_t slot = ((size_t)(j0 + e0 + e) * 2 + (e0 + e == 0)) * Hv + hv;
            v[e] = e0 + e < tab.y ? __ldcg((const float4 *)(a.part_o + (slot * a.rb_rows + q) * DH + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int e = 0; e < SUM_AT; ++e) s.x += v[e].x, s.y += v[e].y, s.z += v[e].z, s.w += v[e].w;
    }
    const int node = rr / a.G;
    const float f = args.scale;
    *(uint2 *)((bf16 *)args.dq + ((size_t)b * a.N + node) * a.qs + (size_t)(g * a.G + rr - node * a.G) * DH + c) =
        live ? make_uint2(pack_bf16(s.x * f, s.y * f), pack_bf16(s.z * f, s.w * f)) : make_uint2(0, 0);
}

bool make_layout(const TreeArgs &a, int rb_rows, bool nodes, bool eight, Layout *lay) {
    const int tab = (4 * a.B + 1) * 4;
    lay->off_tab = OFF_FRONT;
    lay->off_q = (OFF_FRONT + tab + 15) & ~15;
    const int rows = (rb_rows + 15) & ~15;
    lay->off_do = lay->off_q + rows * STAGE_ROW;
    lay->off_n = lay->off_do + rows * STAGE_ROW;
    lay->off_ds = (lay->off_n + (nodes ? (int)sizeof(Nodes) : 0) + 1023) & ~1023;
    lay->off_kn = lay->off_ds + (nodes ? DS_BYTES : 0);
    const int at = lay->off_kn + (nodes ? 2 * KN_BYTES : 0);
    int left = SMEM_MAX - 1024 - at;
    lay->nr = 0;
    if (eight) {
        // two slots of K and one of V, then rings of codes, which cover the copies' latency, then more slots
        const int k_slot = SLOT + SCALES;
        lay->nk = 2, lay->nv = 1;
        left -= 2 * k_slot + SLOT;
        while (lay->nr < 4 && left >= RAW) ++lay->nr, left -= RAW;
        if (lay->nr < 2) return false;
        if (left >= SLOT) ++lay->nv, left -= SLOT;
        if (left >= k_slot) ++lay->nk, left -= k_slot;
        while (lay->nr < MAX_RING && left >= RAW) ++lay->nr, left -= RAW;
    } else {
        const int slots = left / SLOT;
        if (slots < 3) return false;
        lay->nv = slots / 2 < MAX_RING ? slots / 2 : MAX_RING;  // (K is held until dQ has read it)
        lay->nk = slots - lay->nv < MAX_RING ? slots - lay->nv : MAX_RING;
    }
    lay->off_k = at;
    lay->off_v = lay->off_k + lay->nk * SLOT;
    lay->off_sc = lay->off_v + lay->nv * SLOT;
    lay->off_raw = lay->off_sc + (eight ? lay->nk * SCALES : 0);
    lay->smem = lay->off_raw + lay->nr * RAW + 1024;
    return lay->smem <= SMEM_MAX;
}

// The fewest row blocks whose shared memory fits (0: none; the rings of 8-bit codes and a table of thousands of
// sequences leave no room for 128 rows).
int row_blocks(const TreeArgs &a) {
    Layout lay;
    for (int n = ceil_div(a.R, ROWS); n <= ceil_div(a.R, 32); ++n)
        if (make_layout(a, ceil_div(a.R, n), n == 1 && a.N <= MAX_NODES, a.cache.dtype == SP_E4M3, &lay)) return n;
    return 0;
}

template <bool NODES, bool EIGHT>
cudaError_t run(const TreeBackArgs &a, const Layout &lay, const CUtensorMap &mk, const CUtensorMap &mv, int2 *tab, cudaStream_t st) {
    static bool known[MAX_DEVICES] = {};
    const cudaError_t e = allow_smem(tree_back_tc_kernel<NODES, EIGHT>, SMEM_MAX, known);
    if (e != cudaSuccess) return e;
    return launch_k(tree_back_tc_kernel<NODES, EIGHT>, dim3(a.t.plan.tc_ctas), dim3(THREADS), (size_t)lay.smem, st, mk, mv, a, lay, tab);
}

}  // namespace

bool tree_back_tc_supported(const TreeArgs &a) {
    const bool eight = a.cache.dtype == SP_E4M3;
    return a.dh == DH && a.dtype == SP_BF16 && (a.cache.dtype == SP_BF16 || eight) && a.B <= MAX_B && row_blocks(a) > 0 &&
           (eight || a.cache.kv.layout == SP_KV_CONTIGUOUS || (long long)a.cache.kv.n_pages * a.Hkv * a.cache.kv.page_size <= 0x7fffffffLL);
}

void plan_tree_back_tc(TreeArgs *a, int n_sm) {
    a->n_rb = row_blocks(*a);
    a->rb_rows = ceil_div(a->R, a->n_rb);
    const int Hv = a->Hkv * a->n_rb;
    // (the tile list's numbers stay below 2^30)
    const long long most = (long long)((1 << 30) / a->B - 1) * TILE;
    if (a->most_len > most) a->most_len = (int)most;
    AttnArgs &p = a->plan;
    p.B = a->B;
    p.tc_ctas = attn_tc_ctas(n_sm, Hv);
    if (p.tc_ctas / Hv > MAX_GRP) p.tc_ctas = MAX_GRP * Hv;
    p.tc_min_tiles = kBackMinTiles;
    p.tc_seg_cost = kBackSegCost;
    p.tc_merge_kernel = 1;
}

int tree_back_tc_groups(const TreeArgs &a) { return a.plan.tc_ctas / (a.Hkv * a.n_rb); }
size_t tree_back_tc_slots(const TreeArgs &a) { return 2 * (size_t)a.plan.tc_ctas; }

cudaError_t launch_tree_back_tc(const TreeBackArgs &args, int2 *split_tab, cudaStream_t st) {
    const TreeArgs &a = args.t;
    Layout lay;
    const bool nodes = a.n_rb == 1 && a.N <= MAX_NODES, eight = a.cache.dtype == SP_E4M3;
    if (!make_layout(a, a.rb_rows, nodes, eight, &lay)) return cudaErrorInvalidValue;
    CUtensorMap mk, mv;
    memset(&mk, 0, sizeof mk);
    memset(&mv, 0, sizeof mv);
    if (a.cache.kv.layout == SP_KV_PAGED && !eight) {
        const long long blocks = (long long)a.cache.kv.n_pages * a.Hkv;
        if (!encode_kv_pages_bf16(&mk, a.cache.kv.k_pool, blocks, a.cache.kv.page_size) ||
            !encode_kv_pages_bf16(&mv, a.cache.kv.v_pool, blocks, a.cache.kv.page_size))
            return cudaErrorInvalidValue;
    }
    cudaError_t e = nodes ? cudaSuccess : launch_tree_back_rows_tc(args, st);
    if (e != cudaSuccess) return e;
    const auto go = eight ? nodes ? run<true, true> : run<false, true> : nodes ? run<true, false> : run<false, false>;
    e = go(args, lay, mk, mv, split_tab, st);
    if (e != cudaSuccess) return e;
    return launch_k(tree_back_tc_sum_kernel, dim3(a.Hkv * a.n_rb, tree_back_tc_groups(a), ceil_div(a.rb_rows, SUM_ROWS)),
                    dim3(SUM_THREADS), 0, st, args, (const int2 *)split_tab, (int)!nodes);
}

}  // namespace sp

// Attention of a drafted tree over [cache ; tree] (Eq. 1-3, the causal part replaced
// by the tree's masks) on tcgen05 tensor cores: head_dim 128, bf16 rows, caches of
// bf16 or of 8-bit codes with a scale per (token, kv head).
//
// Work: the cached tokens of every sequence are cut into tiles of 128, a tile for its
// nodes behind them; the list of all sequences' tiles is cut into shares as in
// sp_attn_plan.cuh, and CTA (share, kv head, row block) walks its share; a share's piece
// of one sequence is a segment.  A pair that lies inside one share is finished there,
// the others leave partials that a second kernel merges in share order.
//
// The G N query rows of a kv head are the MMA's M side:
//   up to 128 rows: one M tile.  With at most 64 (32) rows the tile holds 2 (4) copies
//     of them, and copy c keeps the weights of its own 64 (32) tokens of each key tile and
//     zeros elsewhere: the exponentials of few rows spread over all four SM sub-partitions
//     (a row is otherwise one thread's work), the product costs what it cost, and the
//     copies are added up once a segment.  Two pipelines take alternate key tiles, each
//     with its own scores, softmax warpgroup and output accumulator.
//   up to 256 rows: two M tiles, one a pipeline, both over every key tile.
//   more: row blocks, as further CTAs.
// Per key tile and pipeline:
//   S = Q K^T     128 x 128, Q in shared memory.  bf16: as they are.  8-bit codes enter
//                 the product as they are (kind::f8f6f4); q is the sum of two 8-bit
//                 parts, exact to 2^-18 of the row's largest element, and the token's and
//                 the row's scales multiply the score
//   softmax       a row a thread, the running max moved only when it grows by 2^8
//   O += P V      P over the first half of S in TMEM.  bf16, or, for 8-bit caches, 16-bit
//                 floats against V's codes as 16-bit floats (exact); V's scale joins the
//                 exponent, w = 2^(x + log2 v_scale - m), so that w <= 2^8 whatever the
//                 scales, and the row sum takes w / v_scale
// The nodes' own keys never lose to the cache's format: bf16 nodes are copied, and for an
// 8-bit cache their keys are two 8-bit parts in the two halves of the tile, added up in the
// same scores (to 2^-18 of a key's largest element), their values 16-bit floats (exact but for
// elements below 2^-24 of a value's largest).
// What a row does not see: scores are replaced by -inf (not added to), rows of a tile past
// the sequence's end are zeros, and a node's non-finite values are taken out of the
// product and added afterwards to the rows that see the node.  What it does see: NaN scores
// leave a sum of NaN (in a part with no other score the least finite max stands for theirs), a
// weight that vanishes beside the row's max is never 0 where parts are added, and dims that
// come out infinite or NaN are made of the cached values again (bf16; 8-bit caches hold no
// infinities).
//
// Warps 0-7: the two softmax warpgroups; then the MMA issuer (it owns TMEM) and the loaders.
// bf16: three warps load queries, two each K and V (TMA boxes of whole pages, cp.async
// elsewhere).  8-bit: two warps load K, one V's codes as they lie and the scales, and four turn
// these into 16-bit floats and the softmax's constants, and load the queries.  Every wait is
// time-limited (SP_DEV_TIMEOUT).
//
// What bounds it, with the merge:
//   bf16          HBM.  64 sequences of 1024 to 8192 tokens, 32 query heads, 8 kv heads, 16
//                 nodes: 210 to 220 us, 5.6 to 5.9 TB/s.  One sequence of 2048 tokens, 8 nodes:
//                 15.6 to 16.2 us, of which 2.7 to know the shares, 2 to the first scores, 1.6
//                 for an epilogue and 4 for the merge and its launch
//   8-bit         the chain of a pipeline, scores -> softmax -> product -> next scores (half of
//                 TMEM is scores, half outputs: no room for the next scores before the product
//                 has read the weights).  8 sequences of 32768 tokens, 40 heads, 32 nodes (160
//                 rows, two M tiles): 377 us, 0.46 PFLOP/s, some 5000 cycles of softmax in 6800
//                 a tile.  128 sequences of 300 to 4000 tokens, 32 heads, one node: 185 to 196 us,
//                 3.0 TB/s, 2600 cycles a tile that the conversion, the V loader and the MMA issuer
//                 fill to 60 - 80 %.
// The kernel's code is as large as what the instruction caches hold: loops are unrolled as
// little as their latency allows (unrolling the conversion and the loaders from 95 to 105 KB of
// code took the 128 sequences from 287 to 378 us), and waits are few instructions.
#include <cudaTypedefs.h>
#include <float.h>
#include <string.h>

#include "sp_attn_plan.cuh"
#include "sp_cache.cuh"
#include "sp_gemm.cuh"
#include "sp_sm100.cuh"

namespace sp {

namespace {

constexpr int TILE = 128;                       // tokens of a key tile
constexpr int SLOT16 = TILE * DH * 2;           // K or V of a tile in 16 bits, 32 KB
constexpr int SLOT8 = TILE * DH;                // in 8 bits, 16 KB
constexpr int PARAMS = 3 * TILE * 4;            // k scales and log2 v scales by pairs, 1 / v scale
constexpr int Q_TILE = 128 * DH * 2;            // an M tile of queries: bf16, or two 8-bit parts
constexpr int CONV = 2;                         // converted V slots
constexpr int MAX_RING = 8, MAX_AHEAD = 3;     // slots of a ring; tiles that V and scales are copied ahead
constexpr int SMEM_MAX = 227 * 1024;
constexpr int SOFT = 256;                       // softmax threads
constexpr int BAR_EPI = 1, BAR_WG = 2;          // (BAR_WG + 1: the second warpgroup's)
constexpr uint32_t O_COL = 256;                 // TMEM: S0 S1 [0, 256), O0 O1 [256, 512)
// Fewest tiles a share holds on average (one sequence of 2048 tokens, 8 kv heads: 26.1, 20.1,
// 21.0, 21.4 us with 1, 2, 3, 4), and the cost of a segment in tiles (200 sequences of 50 to 600
// tokens, 8-bit: 109, 109, 112, 113 us with 2, 3, 4, 6; long ones 195, 195, 194, 197).
constexpr int kTreeMinTiles = 2;
constexpr int kTreeSegCost = 3;

struct Layout {
    int nk, nv;                                 // ring slots
    int off_q, off_k, off_v, off_c, off_st, off_sc, off_tab;  // (off_c: converted V, then its
                                                // constants; off_st: staging of the copies'
                                                // parts; off_sc: of the scales)
    int smem;
};

struct Bars {
    uint64_t k_full[MAX_RING], k_empty[MAX_RING], v_full[MAX_RING], v_empty[MAX_RING];
    uint64_t c_full[CONV], c_empty[CONV], c_par[CONV];
    uint64_t s_full[2], p_full[2], pv_done, q_full, q_empty, fin;
    unsigned long long vbad[MAX_RING][4];       // nodes with non-finite values, by V slot and warp
    unsigned long long seg_vbad;
    unsigned odd_dims[3][DH / 32];              // dims with +inf, -inf, NaN among a segment's cached values
    int odd_cached;                             // a row of the segment came out infinite or NaN
    uint32_t tmem;
    int abort;
    int wsum[32];
};
constexpr int OFF_ML = 1024;                    // (max, sum) of [pipeline][lane]
constexpr int OFF_L = OFF_ML + 2 * 128 * 8;      // 1 / sum of [warpgroup][row]
constexpr int OFF_SEES = OFF_L + 2 * 128 * 4;   // nodes that a row sees, [segment parity][row]
constexpr int OFF_RS = OFF_SEES + 2 * 256 * 8;  // scale of a row's 8-bit queries, the same
constexpr int OFF_CUTS = OFF_RS + 2 * 256 * 4;
constexpr int OFF_FRONT = OFF_CUTS + (MAX_GRP + 4) * 4;
static_assert(sizeof(Bars) <= OFF_ML, "barrier block");

// Warp roles: softmax 0-7, MMA 8; bf16 caches: queries 9-11, producers 12-15; 8-bit caches:
// K producers 9-10, V's codes and scales 11, converters 12-15 (values, constants, queries).
constexpr int THREADS = 512;
constexpr int MMA = 8, V_CODES = 11, CVT = 12, CVT_WARPS = 4;
template <bool E4>
struct Roles {
    static constexpr int K_WARP = E4 ? 9 : 12, V_WARP = K_WARP + 2, V_WARPS = E4 ? 0 : 2;  // producers
    static constexpr int Q_WARP = E4 ? CVT : 9, Q_WARPS = E4 ? CVT_WARPS : 3;              // load the queries
    // Registers a thread: the softmax warps take what the other roles leave of the launch's
    // 128 (8 x 136 + 8 x 120 = 8 x 160 + 8 x 96 = 16 x 128 a lane).  With 128 everywhere 50 to
    // 350 bytes a thread spill, more in all than the L1 that the shared memory leaves holds: a
    // reload then waits for the L2 behind the cache stream.
    static constexpr int SOFT_REGS = E4 ? 136 : 160, OTHER_REGS = E4 ? 120 : 96;
};
template <int N>
__device__ __forceinline__ void regs_inc() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_dec() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
// mbar_wait by a whole warp with one verdict, in few instructions: the kernel waits in some
// twenty places and its loops have to stay in the instruction cache.
__device__ __forceinline__ bool wait_warp(uint64_t *bar, uint32_t parity, volatile int *abort) {
    bool done = mbar_try_wait(bar, parity);
    if (!__all_sync(0xffffffffu, done)) {
        const uint64_t t0 = global_ns();
#pragma unroll 1
        while (!done) {
            done = mbar_try_wait(bar, parity);
            if (!done && (*abort || global_ns() - t0 > kWaitLimitNs)) {
                *abort = 1;
                break;
            }
        }
    }
    return __all_sync(0xffffffffu, done);
}
// One arrival of a warp whose lanes have all done their part.
__device__ __forceinline__ void arrive_warp(uint64_t *bar, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
}

// ---- TMEM accesses without a wait behind every one ----------------------------
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
// Earlier loads complete; 32 of their values are named so that no use moves in front.
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
template <int N>
__device__ __forceinline__ void load_cols(uint32_t addr, float (&v)[N]) {  // N columns, complete
    static_assert(N == 32 || N == 64, "");
    ld32_async(addr, v);
    if constexpr (N == 64) ld32_async(addr + 32, v + 32);
    ld_wait(v);
    if constexpr (N == 64) ld_wait(v + 32);
}
__device__ __forceinline__ void st16_async(uint32_t addr, const float *v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
        "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]),
        "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
        : "memory");
}
template <int W>
__device__ __forceinline__ void tmem_ldw(uint32_t addr, float (&v)[W]) {
    static_assert(W == 16, "");
    tmem_ld16(addr, v);
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void zero16_async(uint32_t addr) {
    const float z[16] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    st16_async(addr, z);
}

// ---- two fp32 operations an instruction ----------------------------------------
__device__ __forceinline__ void fma2(float &d0, float &d1, float a0, float a1, float b0, float b1, float c0, float c1) {
    asm("{\n\t.reg .b64 a, b, c, d;\n\t"
        "mov.b64 a, {%2, %3};\n\t"
        "mov.b64 b, {%4, %5};\n\t"
        "mov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\t"
        "mov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d0), "=f"(d1)
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void mul2(float &d0, float &d1, float a0, float a1, float b0, float b1) {
    asm("{\n\t.reg .b64 a, b, d;\n\t"
        "mov.b64 a, {%2, %3};\n\t"
        "mov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 d, a, b;\n\t"
        "mov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d0), "=f"(d1)
        : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}

// D[tmem] (+)= A[smem] * B[smem]^T on 8-bit elements (32 of K), issued by one thread.
__device__ __forceinline__ void mma_e4m3(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc));
}
__device__ __forceinline__ void expect_tx(uint64_t *bar, uint32_t bytes) {
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// The tile list: prefix[b] = tiles of the sequences before b, each sequence's cache id,
// length and node count.  By all THREADS threads.
__device__ __forceinline__ void tree_prefix(const TreeArgs &a, int *prefix, int *sids, int *lens, int *nodes, int *wsum,
                                            int *status) {
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
        nodes[b] = checked_nodes(a, n, status);
        const int v = ceil_div(sq.len, TILE) + 1;
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
// Its piece of sequence b.
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

// The key tiles of a share, in order.
struct TileWalk {
    const Share &sh;
    Seg sg;
    int b, i;  // sequence, tile of its piece
    __device__ __forceinline__ explicit TileWalk(const Share &s) : sh(s), b(s.b0), i(0) {
        if (!done()) sg = piece(sh, b);
    }
    __device__ __forceinline__ bool done() const { return b >= sh.b1; }
    __device__ __forceinline__ bool fresh() const { return sg.t_a + i == sg.nt - 1; }  // the nodes' tile
    __device__ __forceinline__ void next() {
        if (++i < sg.n) return;
        i = 0;
        if (++b < sh.b1) sg = piece(sh, b);
    }
};
// Page ids of the tiles that a warp asks for, 32 at a time (lane j: page first + j of
// sequence b).
struct Pages {
    int b = -1, first = 0, ids = 0, bits;
    bool paged;
    __device__ __forceinline__ Pages(bool pg, int P_bits) : bits(P_bits), paged(pg) {}
    // before the rows of sequence b from t0 on are asked for; by the whole warp
    __device__ __forceinline__ void at(const TreeArgs &a, const int *sids, const int *lens, int b_, int t0, int lane) {
        const int lp = t0 >> bits;
        if (!paged || (b == b_ && lp + (TILE >> bits) <= first + 32)) return;
        b = b_;
        first = lp;
        ids = -1;
        if ((long long)(lp + lane) << bits < lens[b] && lp + lane < a.cache.kv.max_pages)
            ids = __ldg(a.cache.kv.page_table + (size_t)sids[b] * a.cache.kv.max_pages + lp + lane);
        if (ids >= a.cache.kv.n_pages) ids = -1;
    }
    // page of row r of the tile (negative: none)
    __device__ __forceinline__ int page(int t0, int r) const {
        return __shfl_sync(0xffffffffu, ids, (t0 >> bits) - first + (r >> bits));
    }
};
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
        "l"(src), "r"(bytes), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void cp_async4(void *dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

// One of four (a loop that stays small over values that were loaded together).
__device__ __forceinline__ uint4 pick(const uint4 (&x)[4], int k) {
    const uint4 a = k & 1 ? x[1] : x[0], b = k & 1 ? x[3] : x[2];
    return k & 2 ? b : a;
}

// 2^k that brings a finite amax from 2^-100 on into [128, 256) (a smaller one: k = 107), as the
// factor and k; both 2^k and 2^-k are normal numbers.
__device__ __forceinline__ float pow2_scale(float amax, int *k) {
    int e = (int)((__float_as_uint(amax) >> 23) & 0xff) - 127;
    e = min(max(e, -100), 127);
    *k = 7 - e;
    return __int_as_float((*k + 127) << 23);
}
__device__ __forceinline__ float pow2i(int k) { return __int_as_float((k + 127) << 23); }

// The two 8-bit parts of 8 scaled values: hi = rn(x), lo = rn(x - hi).
__device__ __forceinline__ void split_codes(const float (&x)[8], uint2 *hi, uint2 *lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[i] = float_to_codes2(x[2 * i], x[2 * i + 1]);
        const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)h[i], __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&r));
        l[i] = float_to_codes2(x[2 * i] - f.x, x[2 * i + 1] - f.y);
    }
    *hi = make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
    *lo = make_uint2(l[0] | l[1] << 16, l[2] | l[3] << 16);
}
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}
// The four codes of a word as 16-bit floats.
__device__ __forceinline__ void codes4_to_half4(uint32_t w, uint32_t *h0, uint32_t *h1) {
    asm("{\n\t.reg .b16 l, u;\n\t"
        "mov.b32 {l, u}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, l;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, u;\n\t}"
        : "=r"(*h0), "=r"(*h1)
        : "r"(w));
}
// A tile's constants: for tokens 2 i, 2 i + 1 their k scales, then log2 of their v scales
// (operand pairs of two-wide instructions); this is token t's k scale.
__device__ __forceinline__ int par_at(int t) { return 4 * (t >> 1) + (t & 1); }
// byte offset of 16-byte chunk c (0..7) of row r of an 8-bit tile (128-byte rows, swizzled)
__device__ __forceinline__ uint32_t off8(int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); }

// The queries of sequence b into the score product's A operand, each copy of a row (dead
// rows: zeros), as bf16 [dim half][row][128 B] or as two 8-bit parts [part][row][128 B], and
// what its softmax thread needs of it: the nodes it sees and the parts' scale.  16 lanes a
// row; the first `rows` of them (an even number) by warps wi of nw.
template <bool E4, int TPC, int MT>
__device__ __forceinline__ void load_queries(const TreeArgs &a, int b, int n, int g, int rb, uint8_t *Q,
                                             unsigned long long *sees, float *scale, int rows, int wi, int nw, int lane) {
    const int c = lane & 15;
    // pairs of rows whose loads are under way together: they wait for one latency (200 sequences
    // of 10 to 16 tokens, 64 nodes, 8-bit, with the nodes' rows likewise: 387 -> 353 us)
    constexpr int AT_ONCE = 4;
#pragma unroll 1
    for (int r1 = wi * 2 + (lane >> 4); r1 < rows; r1 += AT_ONCE * 2 * nw) {
        uint4 ahead[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int r = r1 + k * 2 * nw, rr = rb * a.rb_rows + r, node = rr / a.G;
            ahead[k] = make_uint4(0, 0, 0, 0);
            unsigned long long bits = 0;
            if (r < a.rb_rows && rr < a.R && node < n) {
                ahead[k] = *(const uint4 *)((const bf16 *)a.q + ((size_t)b * a.N + node) * a.qs + (size_t)(g * a.G + rr - node * a.G) * DH + c * 8);
                if (c == 0) bits = tree_mask(a, b, node, n);
            }
            if (c == 0 && r < rows) sees[r] = bits;
        }
#pragma unroll(E4 ? 1 : AT_ONCE)
        for (int k = 0; k < AT_ONCE; ++k) {
            const int r = r1 + k * 2 * nw;
            if (r - (lane >> 4) >= rows) break;
            const uint4 u = E4 ? pick(ahead, k) : ahead[k];  // (8-bit: the code has to stay small)
            uint8_t *q = Q + (MT == 2 ? (r >> 7) * Q_TILE : 0);
            const int rt = MT == 2 ? r & 127 : r;
            if constexpr (!E4) {
#pragma unroll
                for (int k = 0; k < 128 / TPC; ++k)
                    st_shared_v4(q + (c >> 3) * 16384 + off8(k * TPC + rt, c & 7), u.x, u.y, u.z, u.w);
            } else {
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
                float v[8], amax = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[2 * i] = __uint_as_float(w[i] << 16);
                    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                    amax = fmaxf(amax, fmaxf(fabsf(v[2 * i]), fabsf(v[2 * i + 1])));
                }
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                int k2;
                const float f = pow2_scale(amax, &k2);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= f;
                uint2 hi, lo;
                split_codes(v, &hi, &lo);
                if (c == 0) scale[r] = pow2i(-k2) + (amax - amax);  // (an infinite query: NaN)
#pragma unroll
                for (int k = 0; k < 128 / TPC; ++k) {
                    *(uint2 *)(q + off8(k * TPC + rt, c >> 1) + (c & 1) * 8) = hi;
                    *(uint2 *)(q + 16384 + off8(k * TPC + rt, c >> 1) + (c & 1) * 8) = lo;
                }
            }
        }
    }
    fence_proxy_async();  // -> tensor-core reads
}

// The non-finite values of the nodes in `odd` added to what was written for the rows of
// the block that see them: the output, or the partial at part.  A row a thread (rare).
__device__ __forceinline__ void add_non_finite(const TreeArgs &a, int b, int g, int rb, int n, unsigned long long odd,
                                               bool whole, float *part, int q) {
    const int rr = rb * a.rb_rows + q, node = rr / a.G;
    if (q >= a.rb_rows || rr >= a.R || node >= n) return;
    bf16 *out = (bf16 *)a.out + (((size_t)b * a.N + node) * a.Hq + (g * a.G + rr - node * a.G)) * DH;
#pragma unroll 1
    for (unsigned long long left = odd & tree_mask(a, b, node, n); left; left &= left - 1) {
        const bf16 *v = (const bf16 *)a.v_new + ((size_t)b * a.N + (__ffsll(left) - 1)) * a.vs + (size_t)g * DH;
#pragma unroll 1
        for (int d = 0; d < DH; ++d) {
            const float z = to_f(v[d]);
            if (isfinite(z)) continue;
            if (whole) out[d] = __float2bfloat16_rn(to_f(out[d]) + z);
            else part[(size_t)q * DH + d] += z;
        }
    }
}

// Which dims of the cached values of tokens [t, t_end) of head g are not finite, bf16.  16 threads
// a token, 8 dims each (rare).
__device__ __forceinline__ void odd_cached_dims(const CacheDev &c, int sid, int g, int t, int t_end, unsigned (*dims)[DH / 32]) {
    if (t >= t_end) return;
    const uint16_t *v = (const uint16_t *)cache_base(c, sid, 1);
    const int chunk = threadIdx.x & 15, shift = chunk * 8 & 31;
    unsigned up = 0, down = 0, nan = 0;
#pragma unroll 1
    for (t += threadIdx.x >> 4; t < t_end; t += SOFT / 16) {
        long long row;
        int step;
        if (!cache_row(c, sid, t, &row, &step)) continue;
        const uint4 u = *(const uint4 *)(v + (row + (long long)g * step) * DH + chunk * 8);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t x = w[i >> 1] >> (i & 1) * 16 & 0xffffu;
            const unsigned bit = 1u << (shift + i);
            up |= x == 0x7f80u ? bit : 0;
            down |= x == 0xff80u ? bit : 0;
            nan |= (x & 0x7fffu) > 0x7f80u ? bit : 0;
        }
    }
    if (up) atomicOr(&dims[0][chunk >> 2], up);
    if (down) atomicOr(&dims[1][chunk >> 2], down);
    if (nan) atomicOr(&dims[2][chunk >> 2], nan);
}

// n cached rows (`step` bytes apart) into rows r0 .. of a slot in the MMA's layout, 16 bytes
// at a time by 64 threads: zeros if there is no source.  A thread keeps its chunk of the row
// and walks rows 8 (8-bit) or 4 apart, so that addresses advance by constants.
template <bool E4>
__device__ __forceinline__ void copy_rows(uint8_t *dst, int r0, int n, const uint8_t *src, size_t step, bool have, int t) {
    constexpr int CH = E4 ? 8 : 16, APART = 64 / CH;
    const int c = t & (CH - 1), r = t / CH;
    src += (size_t)r * step + c * 16;
    const size_t hop = step * APART;
#pragma unroll 4
    for (int i = r; i < n; i += APART, src += hop) {
        uint8_t *d = dst + (E4 ? off8(r0 + i, c) : kv_off(r0 + i, c));
        if (have) cp_async16(d, src);
        else st_shared_v4(d, 0, 0, 0, 0);
    }
}

// ---------------------------------------------------------------------------
// TPC: rows of a copy, and tokens of a tile that a copy weighs (32, 64, 128); MT: M tiles.
template <bool E4, int TPC, int MT>
__global__ void __launch_bounds__(THREADS, 1)
    tree_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                   const __grid_constant__ TreeArgs a, const __grid_constant__ Layout lay, int2 *split_tab) {
    typedef Roles<E4> Ro;
    constexpr int NC = 128 / TPC;  // copies
    static_assert(MT == 1 || TPC == 128, "two M tiles hold one copy each");
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    Bars *bars = (Bars *)smem;
    float2 *ml_s = (float2 *)(smem + OFF_ML);
    float *l_s = (float *)(smem + OFF_L);
    int *cuts = (int *)(smem + OFF_CUTS);
    volatile int *abort = &bars->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int B = a.B, Hkv = a.Hkv, Hv = Hkv * a.n_rb;
    int *prefix = (int *)(smem + lay.off_tab), *sids = prefix + B + 1, *lens = sids + B, *nodes = lens + B;
    // rows of a segment's queries that are loaded; the others, and what belongs to them, are
    // cleared with the first two segments (two buffers) and stay so
    const int live_rows = (a.rb_rows + 1) & ~1;
    const bool paged = a.cache.kv.layout == SP_KV_PAGED;
    const int P = a.cache.kv.page_size, P_bits = 31 - __clz(max(P, 1));  // 16, 32 or 64 (0 contiguous)
    constexpr int ROW = DH * (E4 ? 1 : 2);  // bytes of a cached row
    // the first kernel of its call: nothing of the caller's is read before
    pdl_wait();

    tree_prefix(a, prefix, sids, lens, nodes, bars->wsum, blockIdx.x == 0 ? a.status : nullptr);
    const int T = prefix[B];
    const int n_grp = share_count((int)gridDim.x / Hv, T, B, a.plan.tc_min_tiles);
    const int grp = blockIdx.x / Hv, hv = blockIdx.x - grp * Hv, g = hv / a.n_rb, rb = hv - g * a.n_rb;
    if (grp >= n_grp) return;  // uniform over the CTA: no share
    if (threadIdx.x < PLAN_THREADS) build_cuts(a.plan, prefix, T, n_grp, cuts, bars->wsum);
    if (threadIdx.x == THREADS - 1) {
#pragma unroll 1
        for (int i = 0; i < lay.nk; ++i) {
            mbar_init(&bars->k_full[i], 64);
            mbar_init(&bars->k_empty[i], 1);
        }
#pragma unroll 1
        for (int i = 0; i < lay.nv; ++i) {
            mbar_init(&bars->v_full[i], 64);  // two warps; 8-bit: one, twice a lane
            mbar_init(&bars->v_empty[i], E4 ? CVT_WARPS : 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars->c_full[i], CVT_WARPS);
            mbar_init(&bars->c_par[i], CVT_WARPS);
            mbar_init(&bars->c_empty[i], 1);
            mbar_init(&bars->s_full[i], 1);
            mbar_init(&bars->p_full[i], 4);
        }
        mbar_init(&bars->q_full, Ro::Q_WARPS);
        mbar_init(&bars->q_empty, 1 + SOFT / 32);
        mbar_init(&bars->pv_done, 1);
        mbar_init(&bars->fin, 1);
        bars->abort = 0;
        bars->odd_cached = 0;
        fence_mbar_init();
        if (paged) {
            prefetch_tmap(&map_k);
            if (!E4) prefetch_tmap(&map_v);
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
        regs_inc<Ro::SOFT_REGS>();
        // ------------------------------------------------------------ softmax + epilogue
        const int wg = warp >> 2, ln = threadIdx.x & 127;  // pipeline; TMEM lane
        const int cp = ln / TPC, row_t = ln - cp * TPC;    // copy, row of the M tile
        const int r = (MT == 2 ? wg * 128 : 0) + row_t;    // row of this CTA's block
        const int rr = rb * a.rb_rows + r;                 // query row of the kv head
        const bool active = r < a.rb_rows && rr < a.R;
        const bool warp_active = __any_sync(0xffffffffu, active);
        const uint32_t lane_base = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_col = lane_base + (uint32_t)(wg * 128), o_col = lane_base + O_COL + (uint32_t)(wg * DH);
        bool ok = true;
        uint32_t ks_ph = 0, seg_ph = 0;
        Ring rv(E4 ? CONV : lay.nv);
#pragma unroll 1
        for (int b = sh.b0; b < sh.b1; ++b) {
            int n_tiles, last;  // tiles; the nodes' tile, if it is here
            int left;           // cached tokens from the segment's start on
            {
                const Seg sg = piece(sh, b);  // (the epilogue finds it again)
                n_tiles = sg.n;
                last = sg.nt - 1 - sg.t_a;
                left = lens[b] - sg.t_a * TILE;
            }
            // this segment's queries are there, and with them what the row sees and its scale
            ok = ok && wait_warp(&bars->q_full, seg_ph, abort);
            // (the next ones may come once every softmax warp has seen these and their scores
            // are done: the scores alone run ahead by a whole short segment)
            arrive_warp(&bars->q_empty, lane);
            const int row_s = (int)seg_ph * 256 + r;
            const float rs = E4 ? ((volatile float *)(smem + OFF_RS))[row_s] : 1.f;
            // ---- tiles
            float m = -INFINITY, l = 0.f;
            bool first = true;
#pragma unroll 1
            for (int i = 0; i < n_tiles; ++i, rv.next()) {
                if (MT == 1 && (i & 1) != wg) continue;
                const bool is_fresh = i == last;
                const int n_tok = is_fresh ? 0 : min(TILE, left - i * TILE);
                // warp-uniform verdicts: the TMEM loads and stores are warp-collective
                ok = ok && wait_warp(&bars->s_full[wg], ks_ph, abort);
                // (8-bit: the tile's constants; the nodes' tile: which nodes are not finite)
                if constexpr (E4) ok = ok && wait_warp(&bars->c_par[rv.slot], rv.ph, abort);
                else if (is_fresh) ok = ok && wait_warp(&bars->v_full[rv.slot], rv.ph, abort);
                ks_ph ^= 1;
                if (!ok) continue;
                tc_fence_after();
                if (is_fresh && ln == 0) {  // (the segment's last tile)
                    unsigned long long vb = 0;
#pragma unroll
                    for (int w = 0; w < (E4 ? CVT_WARPS : 2); ++w) vb |= ((volatile unsigned long long *)bars->vbad[rv.slot])[w];
                    bars->seg_vbad = vb;
                }
                if (!warp_active) {  // its lanes' weights reach no row that is used
                    arrive_warp(&bars->p_full[wg], lane);
                    first = false;
                    continue;
                }
                const float *par = (const float *)(smem + lay.off_c + CONV * SLOT16 + rv.slot * PARAMS);
                const bool masked = is_fresh || n_tok < TILE;
                constexpr int CH = TPC == 128 && !E4 ? 64 : 32, N_CH = TPC / CH;  // columns in registers at a time
                const int tok0 = cp * TPC;  // this copy's first token
                // Columns [j0, j0 + CH) of S; 8-bit: in log2 units, with log2 of the value's scale.
                auto scores = [&](int j0, float (&s)[CH]) {
                    load_cols<CH>(s_col + (uint32_t)j0, s);
                    if constexpr (E4) {
                        const float *pj = par + 2 * j0;
#pragma unroll
                        for (int e = 0; e < CH; e += 2) {
                            const float4 p2 = *(const float4 *)(pj + 2 * e);
                            mul2(s[e], s[e + 1], s[e], s[e + 1], rs, rs);
                            fma2(s[e], s[e + 1], s[e], s[e + 1], p2.x, p2.y, p2.z, p2.w);
                        }
                    }
                    if (masked) {
#pragma unroll
                        for (int h = 0; h < CH; h += 32) {
                            const int j = j0 + h;
                            const uint32_t bits =
                                is_fresh ? (j < 64 ? (uint32_t)(((volatile unsigned long long *)(smem + OFF_SEES))[row_s] >> j) : 0u)
                                : n_tok - j >= 32 ? ~0u : n_tok > j ? (1u << (n_tok - j)) - 1u : 0u;
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((bits >> e) & 1)) s[h + e] = -INFINITY;
                        }
                    }
                };
                float s[CH];
                float mt = -INFINITY;
#pragma unroll 1
                for (int c = 0; c < N_CH; ++c) {
                    scores(tok0 + c * CH, s);
                    float mx[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) mx[e] = fmaxf(s[e], s[e + 8]);
#pragma unroll
                    for (int h = 16; h < CH; h += 16)
#pragma unroll
                        for (int e = 0; e < 8; ++e) mx[e] = fmaxf(mx[e], fmaxf(s[h + e], s[h + 8 + e]));
                    mt = fmaxf(mt, fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])),
                                         fmaxf(fmaxf(mx[4], mx[5]), fmaxf(mx[6], mx[7]))));
                    // more than fits the registers: scores go back to where they came from
                    if (N_CH > 1 && (E4 || masked)) {
#pragma unroll
                        for (int h = 0; h < CH; h += 16) st16_async(s_col + (uint32_t)(tok0 + c * CH + h), s + h);
                    }
                }
                if (N_CH > 1 && (E4 || masked)) st_wait();
                if constexpr (!E4) mt *= a.scale_log2;
                const bool grow = mt > m + RESCALE_LOG2 || (m == -INFINITY && mt != -INFINITY);
                const float m_new = grow ? mt : m;
                const float alpha = grow ? (m == -INFINITY ? 0.f : fast_exp2(m - m_new)) : 1.f;
                // (S of this tile was issued behind PV of the pipeline's last one: O is complete)
                if (!first && __any_sync(0xffffffffu, grow)) {
#pragma unroll 1
                    for (int c0 = 0; c0 < DH; c0 += 32) {
                        float o[32];
                        load_cols<32>(o_col + c0, o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] *= alpha;
                        st16_async(o_col + c0, o);
                        st16_async(o_col + c0 + 16, o + 16);
                    }
                    st_wait();
                }
                l *= alpha;
                m = m_new;
                first = false;
                const float mu = m == -INFINITY ? 0.f : m;  // a row that sees nothing: weights of 0
                float ps[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int c = 0; c < N_CH; ++c) {
                    if constexpr (N_CH > 1) load_cols<CH>(s_col + (uint32_t)(tok0 + c * CH), s);
                    float pk[CH / 2];
#pragma unroll
                    for (int e = 0; e < CH; e += 4) {
                        float w[4];
#pragma unroll
                        for (int q = 0; q < 4; q += 2) {
                            if constexpr (E4) add2(w[q], w[q + 1], s[e + q], s[e + q + 1], -mu, -mu);
                            else fma2(w[q], w[q + 1], s[e + q], s[e + q + 1], a.scale_log2, a.scale_log2, -mu, -mu);
                            w[q] = fast_exp2(w[q]);
                            w[q + 1] = fast_exp2(w[q + 1]);
                        }
                        if constexpr (E4) {
                            const float4 iv = *(const float4 *)(par + 2 * TILE + tok0 + c * CH + e);
                            fma2(ps[0], ps[1], w[0], w[1], iv.x, iv.y, ps[0], ps[1]);
                            fma2(ps[2], ps[3], w[2], w[3], iv.z, iv.w, ps[2], ps[3]);
                            pk[e / 2] = __uint_as_float(pack_half(w[0], w[1]));
                            pk[e / 2 + 1] = __uint_as_float(pack_half(w[2], w[3]));
                        } else {
                            add2(ps[0], ps[1], ps[0], ps[1], w[0], w[1]);
                            add2(ps[2], ps[3], ps[2], ps[3], w[2], w[3]);
                            pk[e / 2] = __uint_as_float(pack_bf16(w[0], w[1]));
                            pk[e / 2 + 1] = __uint_as_float(pack_bf16(w[2], w[3]));
                        }
                    }
                    // P over S's first half, whose scores this warp has read (chunk c covers
                    // columns of chunks <= c only)
#pragma unroll
                    for (int h = 0; h < CH / 2; h += 16) st16_async(s_col + (uint32_t)((tok0 + c * CH) / 2 + h), pk + h);
                }
                if constexpr (NC > 1) {  // the other copies' tokens
#pragma unroll
                    for (int z = 0; z < 4; ++z)
                        if (z * 16 < tok0 / 2 || z * 16 >= (tok0 + TPC) / 2) zero16_async(s_col + (uint32_t)(z * 16));
                }
                st_wait();
                l += (ps[0] + ps[1]) + (ps[2] + ps[3]);
                tc_fence_before();
                arrive_warp(&bars->p_full[wg], lane);
            }

            // ---- epilogue: the pipelines' (one M tile) and copies' parts of each row are
            // added; the output (the pair in one share) or a partial is written
            const Seg sg = piece(sh, b);
            const int n = nodes[b];
            const int j_first = group_of(cuts, n_grp, sg.xp), j_last = group_of(cuts, n_grp, sg.xp + sg.nt - 1);
            const bool whole = j_first == j_last;
            const int n1 = MT == 2 ? sg.n : sg.n >> 1;  // tiles of pipeline 1
            // NaN scores alone leave a sum of NaN and no max, which would pass for a part that has
            // seen nothing: the least finite max keeps the sum in what is added up and merged
            if (l != l) m = fmaxf(m, -FLT_MAX);
            ml_s[wg * 128 + ln] = make_float2(m, l);
            named_sync(BAR_EPI, SOFT);
            const bool odd = sg.t_a + sg.n == sg.nt && *(volatile unsigned long long *)&bars->seg_vbad;  // uniform
            float a0, a1 = 0.f, mc, lsum;
            {
                mc = -INFINITY;
                lsum = 0.f;
                if constexpr (MT == 2) {
                    mc = m;
                    lsum = l;
                    a0 = 1.f;
                } else {
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int c = 0; c < NC; ++c) mc = fmaxf(mc, ml_s[p * 128 + c * TPC + row_t].x);
                    const float mu = mc == -INFINITY ? 0.f : mc;
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int c = 0; c < NC; ++c) {
                            const float2 v = ml_s[p * 128 + c * TPC + row_t];
                            if (v.x != -INFINITY) lsum += fast_exp2(v.x - mu) * v.y;
                        }
                    const float m0 = ml_s[ln].x, m1 = ml_s[128 + ln].x;
                    // (0: nothing was seen; a part that vanishes beside the others may hold a NaN)
                    a0 = m0 == -INFINITY ? 0.f : fmaxf(fast_exp2(m0 - mu), kLeastWeight);
                    a1 = m1 == -INFINITY ? 0.f : fmaxf(fast_exp2(m1 - mu), kLeastWeight);
                }
            }
            ok = ok && wait_warp(&bars->pv_done, seg_ph, abort);
            seg_ph ^= 1;
            tc_fence_after();
            // slot of this segment's partial: a share has at most two, the pair that starts
            // in it and the one that began before
            const size_t slot = ((size_t)grp * 2 + (j_first == grp)) * Hv + hv;
            const float inv = lsum == 0.f ? 0.f : 1.f / lsum;
            // where row q of the block goes: the output, or the partial's row
            auto dest = [&](int q, bool *on) {
                const int qr = rb * a.rb_rows + q, nd = qr / a.G;
                *on = nd < n;
                return whole ? (uint8_t *)((bf16 *)a.out + (((size_t)b * a.N + nd) * a.Hq + (g * a.G + qr - nd * a.G)) * DH)
                             : (uint8_t *)(a.part_o + (slot * a.rb_rows + q) * DH);
            };
            float probe = 0.f;  // NaN: a value written is not finite
            auto write = [&](uint8_t *to, bool on, int d, float4 y, float scale) {  // four dims, unnormalised
                if constexpr (!E4) probe = fmaf(y.w, 0.f, fmaf(y.z, 0.f, fmaf(y.y, 0.f, fmaf(y.x, 0.f, probe))));
                if (whole)
                    *(uint2 *)(to + d * 2) = on && scale != 0.f ? make_uint2(pack_bf16(y.x * scale, y.y * scale),
                                                                             pack_bf16(y.z * scale, y.w * scale))
                                                                : make_uint2(0, 0);
                else
                    *(float4 *)(to + d * 4) = y;
            };
            // dims [d, d + W) of this lane's row: both pipelines' parts (one M tile)
            auto parts = [&](int d, auto &o) {
                constexpr int W = sizeof(o) / sizeof(float);
                if (!ok) {
#pragma unroll
                    for (int e = 0; e < W; ++e) o[e] = 0.f;
                } else if constexpr (MT == 2) {
                    tmem_ldw<W>(o_col + d, o);
                } else {
                    float o1[W];
                    tmem_ldw<W>(lane_base + O_COL + d, o);
                    if (n1 > 0) tmem_ldw<W>(lane_base + O_COL + DH + d, o1);
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        // a part without a weight: its accumulator may hold anything
                        const float y0 = a0 != 0.f ? a0 * o[e] : 0.f;
                        o[e] = n1 > 0 && a1 != 0.f ? fmaf(a1, o1[e], y0) : y0;
                    }
                }
            };
            const int d_lo = MT == 2 ? 0 : wg * (DH / 2), d_hi = MT == 2 ? DH : d_lo + DH / 2;
            if constexpr (NC == 1) {
                bool on = false;
                uint8_t *to = active ? dest(r, &on) : nullptr;
#pragma unroll 1
                for (int d = d_lo; d < d_hi; d += 16) {
                    float o[16];
                    parts(d, o);
                    if (active) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4) write(to, on, d + e, make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]), inv);
                    }
                }
            } else {
                // 16 dims of every lane as four swizzled chunks; then (row, chunk) units add the copies
                uint8_t *stage = smem + lay.off_st + wg * 8192;
                if (cp == 0) l_s[wg * 128 + ln] = inv;
#pragma unroll 1
                for (int d = d_lo; d < d_hi; d += 16) {
                    float o[16];
                    parts(d, o);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        st_shared_v4(stage + ln * 64 + ((q ^ ((ln >> 1) & 3)) << 4), __float_as_uint(o[4 * q]),
                                     __float_as_uint(o[4 * q + 1]), __float_as_uint(o[4 * q + 2]), __float_as_uint(o[4 * q + 3]));
                    named_sync(BAR_WG + wg, 128);
#pragma unroll 1
                    for (int it = ln; it < TPC * 4; it += 128) {
                        const int q = it >> 2, c = it & 3;
                        if (q >= a.rb_rows || rb * a.rb_rows + q >= a.R) continue;
                        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int k = 0; k < NC; ++k) {
                            const int lc = k * TPC + q;
                            const float4 v = ld_shared_v4f(stage + lc * 64 + ((c ^ ((lc >> 1) & 3)) << 4));
                            y.x += v.x, y.y += v.y, y.z += v.z, y.w += v.w;
                        }
                        bool on;
                        uint8_t *to = dest(q, &on);
                        write(to, on, d + c * 4, y, l_s[wg * 128 + q]);
                    }
                    named_sync(BAR_WG + wg, 128);
                }
            }
            if (active && cp == 0 && (MT == 2 || wg == 0)) {
                if (!whole) *(float2 *)(a.part_ml + (slot * a.rb_rows + r) * 2) = make_float2(mc, lsum);
                else if (a.lse) store_lse(a, b, rr / a.G, g * a.G + rr % a.G, mc, rr / a.G < n ? lsum : 0.f);
            }
            if (probe != probe) bars->odd_cached = 1;
            tc_fence_before();
            named_sync(BAR_EPI, SOFT);  // both accumulators and ml_s are free, the rows are written
            const bool lost = !E4 && *(volatile int *)&bars->odd_cached;
            if (lost || odd) {  // (uniform, rare)
                if (lost) {
                    // An infinite cached value is NaN where another copy, or a weight that underflows,
                    // has multiplied it by 0.  Every row sees the segment's cached tokens: the dims
                    // that have such values get the sum of them
                    named_sync(BAR_EPI, SOFT);
                    if (threadIdx.x < 3 * (DH / 32)) (&bars->odd_dims[0][0])[threadIdx.x] = 0;
                    if (threadIdx.x == 0) bars->odd_cached = 0;
                    named_sync(BAR_EPI, SOFT);
                    odd_cached_dims(a.cache, sids[b], g, sg.t_a * TILE, min(lens[b], (sg.t_a + sg.n) * TILE), bars->odd_dims);
                    named_sync(BAR_EPI, SOFT);
                    bool on = false;
                    uint8_t *to = nullptr;
                    if (active && cp == 0 && (MT == 2 || wg == 0) && isfinite(lsum) && lsum != 0.f) to = dest(r, &on);
#pragma unroll 1
                    for (int w = 0; on && w < DH / 32; ++w) {
                        const volatile unsigned(*dims)[DH / 32] = bars->odd_dims;
                        const unsigned up = dims[0][w], down = dims[1][w], nan = dims[2][w];
#pragma unroll 1
                        for (unsigned left = up | down | nan; left; left &= left - 1) {
                            const int e = __ffs(left) - 1, d = w * 32 + e;
                            const float z = (nan | (up & down)) >> e & 1 ? NAN : up >> e & 1 ? INFINITY : -INFINITY;
                            if (whole) ((bf16 *)to)[d] = __float2bfloat16_rn(z);
                            else ((float *)to)[d] = z;
                        }
                    }
                }
                if (odd)  // values that were kept out of the product: to the rows that see them
                    add_non_finite(a, b, g, rb, n, *(volatile unsigned long long *)&bars->seg_vbad, whole,
                                   a.part_o + slot * a.rb_rows * DH, threadIdx.x);
                named_sync(BAR_EPI, SOFT);
            }
        }
    } else {
        regs_dec<Ro::OTHER_REGS>();
        if (warp >= Ro::K_WARP && warp < Ro::K_WARP + 2 + Ro::V_WARPS) {
            // ------------------------------------------------------------ producers
            const bool is_v = !E4 && warp >= Ro::V_WARP;
            const int pidx = warp - (is_v ? Ro::V_WARP : Ro::K_WARP), ptid = pidx * 32 + lane;
            const bool lead = pidx == 0;
            uint64_t *full = is_v ? bars->v_full : bars->k_full, *empty = is_v ? bars->v_empty : bars->k_empty;
            const int slot_bytes = E4 ? SLOT8 : SLOT16;
            uint8_t *ring = smem + (is_v ? lay.off_v : lay.off_k);
            const CUtensorMap *map = is_v ? &map_v : &map_k;
            const uint8_t *pool = (const uint8_t *)(is_v ? a.cache.kv.v_pool : a.cache.kv.k_pool);
            const uint64_t pol = policy_evict_first();
            Ring rg(is_v ? lay.nv : lay.nk);
            int bad = 0, filled = 0;
            bool stop = false;
#pragma unroll 1
            for (int b = sh.b0; b < sh.b1 && !stop; ++b) {
                const Seg sg = piece(sh, b);
                const int sid = sids[b], L = lens[b];
                // a contiguous sequence's rows of head g, a token apart
                const uint8_t *seq = nullptr;
                if (!paged && L > 0)
                    seq = (const uint8_t *)(is_v ? a.cache.kv.v_seq : a.cache.kv.k_seq)[sid] + (size_t)g * ROW;
                const size_t seq_step = (size_t)Hkv * ROW;
#pragma unroll 1
                for (int i = 0; i < sg.n; ++i) {
                    const int t = sg.t_a + i, t0 = t * TILE;
                    const bool is_fresh = t == sg.nt - 1;
                    const int n_tok = is_fresh ? 0 : min(TILE, L - t0);
                    const int n_pg = paged ? n_tok >> P_bits : 0;  // whole pages
                    int page = -1;                           // page ids (up to eight), asked for before the wait
                    if (paged && lane * P < n_tok) {
                        const int lp = (t0 >> P_bits) + lane;
                        page = lp < a.cache.kv.max_pages ? a.cache.kv.page_table[(size_t)sid * a.cache.kv.max_pages + lp] : -1;
                        if (page < 0 || page >= a.cache.kv.n_pages) page = -1, bad = 1;
                    }
                    // warp-uniform verdict: the collectives below need every lane
                    if (!wait_warp(&empty[rg.slot], rg.ph ^ 1, abort)) {
                        stop = true;
                        break;
                    }
                    uint8_t *dst = ring + rg.slot * slot_bytes;
                    bool plain = false;  // this thread wrote shared memory or issued cp.async
                    if (n_pg > 0 && lead) {
                        const bool ok = lane < n_pg && page >= 0;
                        const unsigned okm = __ballot_sync(0xffffffffu, ok);
                        if (lane == 0 && okm) expect_tx(&full[rg.slot], __popc(okm) * P * ROW);
                        __syncwarp();
                        if (ok) {  // the cache is read once: evict-first keeps queries and partials in L2
                            const int row = page * Hkv + g;
                            if constexpr (E4) tma_load_2d_hint(dst + lane * P * ROW, map, &full[rg.slot], 0, row * P, pol);
                            else tma_load_4d_hint(dst + lane * P * ROW, map, &full[rg.slot], 0, 0, 0, row * (P / 8), pol);
                        }
                        // a page outside the pool: zeros
#pragma unroll 1
                        for (unsigned miss = ~okm & ((1u << n_pg) - 1u); miss; miss &= miss - 1) {
                            const int j = __ffs(miss) - 1;
#pragma unroll 1
                            for (int e = lane; e < P * ROW / 16; e += 32) st_shared_v4(dst + j * P * ROW + e * 16, 0, 0, 0, 0);
                            plain = true;
                        }
                    }
                    const int r0 = n_pg * (paged ? P : 0);  // first row not covered by TMA
                    if (r0 < n_tok) {
                        plain = true;
                        const uint8_t *src = seq + (size_t)t0 * seq_step;
                        size_t step = seq_step;
                        bool have = true;
                        if (paged) {  // the last, partial page
                            const int pg = __shfl_sync(0xffffffffu, page, n_pg);
                            have = pg >= 0;
                            src = pool + ((size_t)max(pg, 0) * Hkv + g) * P * ROW;
                            step = ROW;
                        }
                        copy_rows<E4>(dst, r0, n_tok - r0, src, step, have, ptid);
                    }
                    // values past the end are multiplied by weights of 0: they must be
                    // finite (keys there give scores that are replaced)
                    if (!E4 && is_v && !is_fresh && n_tok < TILE) {
                        plain = true;
#pragma unroll 1
                        for (int idx = ptid; idx < (TILE - n_tok) * 16; idx += 64)
                            st_shared_v4(dst + kv_off(n_tok + (idx >> 4), idx & 15), 0, 0, 0, 0);
                    }
                    if (is_fresh) {
                        // the nodes' rows: 16 lanes a row, 8 elements a lane (scores of the rows
                        // after the last node's are replaced: of V these rows must be zeros)
                        plain = true;
                        const bf16 *fresh = (const bf16 *)(is_v ? a.v_new : a.k_new) + (size_t)g * DH;
                        const long long fs = is_v ? a.vs : a.ks;
                        const int n = nodes[b], c = lane & 15;
                        unsigned long long vb = 0;
                        // rows whose loads are under way together (bf16: one, its loaders' registers are few)
                        constexpr int AT_ONCE = E4 ? 4 : 1;
                        uint4 some[AT_ONCE];
#pragma unroll 1
                        for (int r = pidx * 2 + (lane >> 4), k = 0; r < (is_v ? 64 : (n + 1) & ~1); r += 4, ++k) {
                            if (k % AT_ONCE == 0) {
#pragma unroll
                                for (int e = 0; e < AT_ONCE; ++e) {
                                    some[e] = make_uint4(0, 0, 0, 0);
                                    if (r + 4 * e < n) some[e] = *(const uint4 *)(fresh + ((size_t)b * a.N + r + 4 * e) * fs + c * 8);
                                }
                            }
                            uint4 u = some[0];
                            if constexpr (E4) u = pick(some, k & 3);
                            uint32_t w[4] = {u.x, u.y, u.z, u.w};
                            if constexpr (!E4) {
                                if (is_v) {
                                    bool odd = false;
#pragma unroll
                                    for (int q = 0; q < 4; ++q) {
                                        const bool lo = (w[q] & 0x7f80u) == 0x7f80u, hi = (w[q] & 0x7f800000u) == 0x7f800000u;
                                        odd = odd || lo || hi;
                                        w[q] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
                                    }
                                    const unsigned o = __ballot_sync(0xffffffffu, odd);
                                    const int even = r & ~1;  // (lanes 0-15 hold the even row)
                                    if (o & 0xffffu) vb |= 1ull << even;
                                    if (o >> 16) vb |= 2ull << even;
                                }
                                st_shared_v4(dst + kv_off(r, c), w[0], w[1], w[2], w[3]);
                            } else {
                                // keys as two 8-bit parts, rows r and 64 + r
                                float v[8];
                                float amax = 0.f;
#pragma unroll
                                for (int q = 0; q < 4; ++q) {
                                    v[2 * q] = __uint_as_float(w[q] << 16);
                                    v[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
                                    amax = fmaxf(amax, fmaxf(fabsf(v[2 * q]), fabsf(v[2 * q + 1])));
                                }
#pragma unroll
                                for (int o = 1; o < 16; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                                int k;
                                const float f = pow2_scale(amax, &k);
#pragma unroll
                                for (int q = 0; q < 8; ++q) v[q] *= f;
                                uint2 hi, lo;
                                split_codes(v, &hi, &lo);
                                *(uint2 *)(dst + off8(r, c >> 1) + (c & 1) * 8) = hi;
                                *(uint2 *)(dst + off8(64 + r, c >> 1) + (c & 1) * 8) = lo;
                            }
                        }
                        if (!E4 && is_v && lane == 0) bars->vbad[rg.slot][pidx] = vb;
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
            if (lead && lane == 0) {
                // drain copies still in flight (only possible after an abort)
                Ring rd(rg.n);
#pragma unroll 1
                for (int j = 0; j < filled; ++j, rd.next())
                    if (j + rg.n >= filled) mbar_wait_drain(&full[rd.slot], rd.ph);
            }
            bad = __any_sync(0xffffffffu, bad);
            if (bad && lane == 0 && a.status) atomicOr(a.status, SP_DEV_BAD_PAGE);
        } else if (E4 && warp >= CVT) {
            // ------------------------------------------------------------ converters
            // V's codes to 16-bit floats in shared memory: 16 codes at a time, eight times a
            // thread and tile (rows r0 + 16 k, chunk c)
            const int ct = threadIdx.x - CVT * 32, cw = warp - CVT;
            const int r0 = ct >> 3, c = ct & 7, flip = c >> 2;
            Ring rv(lay.nv);
            Ring rc(CONV);
            uint32_t seg_ph = 0;
            bool ok = true;
            auto convert = [&](const uint8_t *src, uint8_t *dst) {
                // (the two halves of the chunks in turns: 8 lanes then cover all banks)
                const uint8_t *src0 = src + flip * 8, *src1 = src + 8 - flip * 8;
                uint8_t *to0 = dst + kv_off(r0, 2 * c + flip), *to1 = dst + kv_off(r0, 2 * c + 1 - flip);
#pragma unroll 2
                for (int k = 0; k < 8; ++k) {
                    const uint2 z0 = *(const uint2 *)(src0 + k * 2048), z1 = *(const uint2 *)(src1 + k * 2048);
                    uint32_t h[8];
                    codes4_to_half4(z0.x, &h[0], &h[1]);
                    codes4_to_half4(z0.y, &h[2], &h[3]);
                    codes4_to_half4(z1.x, &h[4], &h[5]);
                    codes4_to_half4(z1.y, &h[6], &h[7]);
                    st_shared_v4(to0 + k * 2 * GROUP_STRIDE, h[0], h[1], h[2], h[3]);
                    st_shared_v4(to1 + k * 2 * GROUP_STRIDE, h[4], h[5], h[6], h[7]);
                }
            };
#pragma unroll 1
            for (TileWalk w(sh); !w.done(); w.next(), rc.next()) {
                const int b = w.b;
                if (w.i == 0) {  // a segment's queries
                    ok = wait_warp(&bars->q_empty, seg_ph ^ 1, abort);
                    if (!ok) break;
                    load_queries<E4, TPC, MT>(a, b, nodes[b], g, rb, smem + lay.off_q, (unsigned long long *)(smem + OFF_SEES) + seg_ph * 256,
                                              (float *)(smem + OFF_RS) + seg_ph * 256, b - sh.b0 < 2 ? TPC * MT : live_rows, cw, CVT_WARPS, lane);
                    arrive_warp(&bars->q_full, lane);
                    seg_ph ^= 1;
                }
                ok = wait_warp(&bars->c_empty[rc.slot], rc.ph ^ 1, abort);
                if (!ok) break;
                uint8_t *dst = smem + lay.off_c + rc.slot * SLOT16;
                float *par = (float *)(smem + lay.off_c + CONV * SLOT16 + rc.slot * PARAMS);
                if (w.fresh()) {
                    if (ct >= 64) par[2 * TILE + ct] = 0.f;  // (weights of 0 are multiplied by these)
                    const int n = nodes[b], c16 = lane & 15;
                    unsigned long long vb = 0;
                    uint4 two_k[2], two_v[2];  // (rows whose loads are under way together)
#pragma unroll 1
                    for (int r = cw * 2 + (lane >> 4), k = 0; r < 64; r += 8, ++k) {
                        if ((r & ~1) >= n) {  // (the pair of rows of this warp)
                            st_shared_v4(dst + kv_off(r, c16), 0, 0, 0, 0);
                            if (c16 == 0) par[2 * TILE + r] = 0.f;
                            continue;
                        }
                        if ((k & 1) == 0) {
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                two_k[e] = two_v[e] = make_uint4(0, 0, 0, 0);
                                if (r + 8 * e < n) {
                                    const size_t row = (size_t)b * a.N + r + 8 * e;
                                    two_k[e] = *(const uint4 *)((const bf16 *)a.k_new + row * a.ks + (size_t)g * DH + c16 * 8);
                                    two_v[e] = *(const uint4 *)((const bf16 *)a.v_new + row * a.vs + (size_t)g * DH + c16 * 8);
                                }
                            }
                        }
                        const uint4 uk = two_k[0], uv = two_v[0];
                        two_k[0] = two_k[1], two_v[0] = two_v[1];
                        const uint32_t wk[4] = {uk.x, uk.y, uk.z, uk.w}, wv[4] = {uv.x, uv.y, uv.z, uv.w};
                        float v[8], amk = 0.f, amv = 0.f;
                        bool odd = false;
#pragma unroll
                        for (int q4 = 0; q4 < 4; ++q4) {
                            amk = fmaxf(amk, fmaxf(fabsf(__uint_as_float(wk[q4] << 16)), fabsf(__uint_as_float(wk[q4] & 0xffff0000u))));
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float y = __uint_as_float(e ? wv[q4] & 0xffff0000u : wv[q4] << 16);
                                const bool fin = isfinite(y);
                                odd = odd || !fin;
                                v[2 * q4 + e] = fin ? y : 0.f;
                                amv = fmaxf(amv, fabsf(v[2 * q4 + e]));
                            }
                        }
#pragma unroll
                        for (int o = 1; o < 16; o <<= 1) {
                            amk = fmaxf(amk, __shfl_xor_sync(0xffffffffu, amk, o));
                            amv = fmaxf(amv, __shfl_xor_sync(0xffffffffu, amv, o));
                        }
                        const unsigned o = __ballot_sync(0xffffffffu, odd);
                        if (o & 0xffffu) vb |= 1ull << (r & ~1);
                        if (o >> 16) vb |= 2ull << (r & ~1);
                        int kk, kv;
                        pow2_scale(amk, &kk);
                        const float f = pow2_scale(amv, &kv);
                        st_shared_v4(dst + kv_off(r, c16), pack_half(v[0] * f, v[1] * f), pack_half(v[2] * f, v[3] * f),
                                     pack_half(v[4] * f, v[5] * f), pack_half(v[6] * f, v[7] * f));
                        if (c16 == 0) {
                            // an infinite key saturates in its parts: its scores are NaN
                            par[par_at(r)] = pow2i(-kk) * a.scale_log2 + (amk - amk);
                            par[par_at(r) + 2] = (float)-kv;
                            par[2 * TILE + r] = pow2i(kv);
                        }
                    }
                    if (lane == 0) bars->vbad[rc.slot][cw] = vb;
                    arrive_warp(&bars->c_par[rc.slot], lane);
                } else {
                    ok = wait_warp(&bars->v_full[rv.slot], rv.ph, abort);
                    if (!ok) break;
                    {  // token ct's constants
                        const float *sc = (const float *)(smem + lay.off_sc) + rv.slot * 2 * TILE + ct;
                        const float floor = 7.888609052210118e-31f;  // 2^-100
                        const float lg = __log2f(sc[TILE] < floor ? floor : sc[TILE]);  // (a NaN stays)
                        par[par_at(ct)] = sc[0] * a.scale_log2;
                        par[par_at(ct) + 2] = lg;
                        par[2 * TILE + ct] = fast_exp2(-lg);  // (a weight times its inverse: lg's error cancels)
                    }
                    arrive_warp(&bars->c_par[rc.slot], lane);
                    convert(smem + lay.off_v + rv.slot * SLOT8 + ct * 16, dst);
                    arrive_warp(&bars->v_empty[rv.slot], lane);
                    rv.next();
                }
                fence_proxy_async();
                arrive_warp(&bars->c_full[rc.slot], lane);
            }
        } else if (E4 && warp == V_CODES) {
            // ------------------------------------------------------------ V's codes and scales
            // as they lie, for the converters; a row of 128 bytes is 8 lanes'
            Ring rg(lay.nv);
            Pages pages(paged, P_bits);
            int filled = 0;
            bool stop = false;
#pragma unroll 1
            for (int b = sh.b0; b < sh.b1 && !stop; ++b) {
                const Seg sg = piece(sh, b);
                const int sid = sids[b], L = lens[b];
                const float *sk = nullptr, *sv = nullptr;
                const uint8_t *v = (const uint8_t *)a.cache.kv.v_pool;
                int t0 = sg.t_a * TILE;
                if (L > 0) {
                    sk = scale_base(a.cache, sid, 0);
                    sv = scale_base(a.cache, sid, 1);
                    if (!paged) v = (const uint8_t *)a.cache.kv.v_seq[sid] + (size_t)(t0 + (lane >> 3)) * (Hkv * ROW) + g * ROW + (lane & 7) * 16;
                }
#pragma unroll 1
                for (const int end = min(L, t0 + sg.n * TILE); t0 < end; t0 += TILE) {
                    const int n_tok = min(TILE, L - t0);
                    pages.at(a, sids, lens, b, t0, lane);
                    if (!wait_warp(&bars->v_empty[rg.slot], rg.ph ^ 1, abort)) {
                        stop = true;
                        break;
                    }
                    uint8_t *dst = smem + lay.off_v + rg.slot * SLOT8;
                    float *sc = (float *)(smem + lay.off_sc) + rg.slot * 2 * TILE + lane;
                    if (paged) {  // a bulk copy a page
                        const int rows = min(P, n_tok - lane * P), pg = pages.page(t0, lane * P);
                        const bool ok = rows > 0 && pg >= 0;
                        const unsigned bytes = __reduce_add_sync(0xffffffffu, ok ? rows * ROW : 0);
                        if (lane == 0 && bytes) expect_tx(&bars->v_full[rg.slot], bytes);
                        __syncwarp();
                        if (ok) {
                            bulk_load(dst + lane * P * ROW, v + ((size_t)pg * Hkv + g) * P * ROW, rows * ROW, &bars->v_full[rg.slot]);
                        } else if (rows > 0) {  // a page outside the pool: zeros
#pragma unroll 1
                            for (int e = 0; e < rows * 8; ++e) st_shared_v4(dst + lane * P * ROW + e * 16, 0, 0, 0, 0);
                        }
#pragma unroll 1
                        for (int r = lane; r < TILE; r += 32, sc += 32) {
                            const int pr = pages.page(t0, r);
                            if (r < n_tok && pr >= 0) {
                                const size_t at = ((size_t)pr * Hkv + g) * P + (r & (P - 1));
                                cp_async4(sc, sk + at);
                                cp_async4(sc + TILE, sv + at);
                            } else {
                                sc[0] = sc[TILE] = 0.f;
                            }
                        }
                    } else {  // (a bulk copy a row took 60 cycles to issue each)
                        const size_t hop = (size_t)(4 * Hkv) * ROW;
                        uint8_t *d = dst + lane * 16;
#pragma unroll 4
                        for (int r = lane >> 3; r < n_tok; r += 4, v += hop, d += 512) cp_async16(d, v);
                        size_t at = (size_t)(t0 + lane) * Hkv + g;
#pragma unroll 1
                        for (int k = 0; k < 4; ++k, at += 32 * Hkv)
                            if (lane + 32 * k < n_tok) {
                                cp_async4(sc + 32 * k, sk + at);
                                cp_async4(sc + TILE + 32 * k, sv + at);
                            } else {  // (weights of 0 are multiplied by what is made of these)
                                sc[32 * k] = sc[TILE + 32 * k] = 0.f;
                            }
                    }
                    // past the end: weights of 0 times zeros
#pragma unroll 1
                    for (int e = n_tok * 8 + lane; e < TILE * 8; e += 32) st_shared_v4(dst + e * 16, 0, 0, 0, 0);
                    fence_proxy_async();
                    cp_async_mbar_arrive(&bars->v_full[rg.slot]);
                    mbar_arrive(&bars->v_full[rg.slot]);  // (the zeros)
                    ++filled;
                    rg.next();
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");  // nothing lands after the CTA is gone
            if (lane == 0) {                                  // (bulk copies: only after an abort)
                Ring rd(lay.nv);
#pragma unroll 1
                for (int j = 0; j < filled; ++j, rd.next())
                    if (j + lay.nv >= filled) mbar_wait_drain(&bars->v_full[rd.slot], rd.ph);
            }
        } else if (!E4 && warp >= Ro::Q_WARP && warp < Ro::Q_WARP + Ro::Q_WARPS) {
            // ------------------------------------------------------------ queries
            uint32_t seg_ph = 0;
#pragma unroll 1
            for (int b = sh.b0; b < sh.b1; ++b, seg_ph ^= 1) {
                if (!wait_warp(&bars->q_empty, seg_ph ^ 1, abort)) break;
                load_queries<E4, TPC, MT>(a, b, nodes[b], g, rb, smem + lay.off_q,
                                          (unsigned long long *)(smem + OFF_SEES) + seg_ph * 256, nullptr,
                                          b - sh.b0 < 2 ? TPC * MT : live_rows, warp - Ro::Q_WARP, Ro::Q_WARPS, lane);
                arrive_warp(&bars->q_full, lane);
            }
        } else if (warp == MMA) {
            // ------------------------------------------------------------ MMA issue
            // Items q of a segment in order: pipeline q & 1, on tile q (one M tile) or q / 2
            // (two).  S of the first two, then PV of item q once its softmax is done and S of
            // item q + 2 into the buffer that softmax has read.  One issuer: it sees every use
            // of every ring slot in order.  (Two, each waiting for its own tiles only, may ask
            // for a slot's next use before the one in between, the other's, has landed; the
            // barrier's parity then answers for the use before that.)  By the whole warp, the
            // instructions under `on` (see elect_one).
            const bool on = elect_one();
            constexpr uint32_t idesc_s = E4 ? (1u << 4) | ((uint32_t)(TILE >> 3) << 17) | (8u << 24) : idesc_bf16_f32(128, TILE);
            constexpr uint32_t idesc_s64 = (1u << 4) | ((uint32_t)(64 >> 3) << 17) | (8u << 24);
            // 16-bit floats: format bits 0 instead of bf16's 1
            constexpr uint32_t idesc_o = E4 ? (1u << 4) | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | (8u << 24)
                                            : idesc_bf16_f32_bmn(128, DH);
            const uint64_t dq0 = sw128_kmajor_desc(smem + lay.off_q);
            const uint64_t dk0 = sw128_kmajor_desc_sbo(smem + lay.off_k, E4 ? 1024 : GROUP_STRIDE);
            const uint64_t dv0 = sw128_mnmajor_desc2(smem + (E4 ? lay.off_c : lay.off_v), HALF_STRIDE, GROUP_STRIDE);
            uint64_t *vf = E4 ? bars->c_full : bars->v_full, *ve = E4 ? bars->c_empty : bars->v_empty;
            Ring rk(lay.nk), rv(E4 ? CONV : lay.nv);
            bool ok = true;
            uint32_t kp = 0;  // phases of p_full, a bit a pipeline
            int j = 0;
            auto issue_s = [&](int q, bool last_s, bool nodes_tile) {
                const int w = q & 1;
                ok = ok && wait_warp(&bars->k_full[rk.slot], rk.ph, abort);
                if (!ok) return;
                tc_fence_after();
                fence_proxy_async();  // cp.async data -> tensor-core reads
                const uint64_t dk = dk0 + (uint32_t)(rk.slot * ((E4 ? SLOT8 : SLOT16) >> 4));
                const uint64_t dq = dq0 + (uint32_t)(MT == 2 ? w * (Q_TILE >> 4) : 0);
                const uint32_t d = tmem + (uint32_t)(w * 128);
                if (on) {
                    if constexpr (E4) {
                        // the nodes' tile: 64 columns, the keys' two parts added in them
                        const uint32_t id = nodes_tile ? idesc_s64 : idesc_s;
#pragma unroll 1
                        for (int part = 0; part < (nodes_tile ? 2 : 1); ++part)
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk)  // part kk / 4 of the queries, 32 dims each
                                mma_e4m3(d, dq + (uint64_t)((kk >> 2) * (16384 >> 4) + (kk & 3) * 2),
                                         dk + (uint64_t)(part * (8192 >> 4) + (kk & 3) * 2), id, kk > 0 ? 1u : (uint32_t)part);
                    } else {
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk)  // 16 dims: 32 B of a row of dim half kk / 4
                            mma_bf16(d, dq + (uint64_t)((kk >> 2) * (16384 >> 4) + (kk & 3) * 2),
                                     dk + (uint64_t)((kk >> 2) * (HALF_STRIDE >> 4) + (kk & 3) * 2), idesc_s, kk > 0);
                    }
                    if (MT == 1 || w) mma_commit(&bars->k_empty[rk.slot]);
                    mma_commit(&bars->s_full[w]);
                    if (last_s) mma_commit(&bars->q_empty);  // (the segment's last scores)
                }
                __syncwarp();
                if (MT == 1 || w) rk.next();
            };
#pragma unroll 1
            for (int b = sh.b0; ok && b < sh.b1; ++b, ++j) {
                const Seg sg = piece(sh, b);
                // the same in every lane, and known to be
                const int items = __shfl_sync(0xffffffffu, sg.n, 0) * MT;
                const bool has_fresh = __shfl_sync(0xffffffffu, (int)(sg.t_a + sg.n == sg.nt), 0);
                if (!wait_warp(&bars->q_full, (uint32_t)(j & 1), abort)) break;
#pragma unroll 1
                for (int q = -2; ok && q < items; ++q) {
                    if (q >= 0) {
                        const int w = q & 1;
                        ok = wait_warp(&vf[rv.slot], rv.ph, abort) && wait_warp(&bars->p_full[w], (kp >> w) & 1, abort);
                        if (!ok) break;
                        kp ^= 1u << w;
                        tc_fence_after();
                        fence_proxy_async();
                        const uint64_t dv = dv0 + (uint32_t)(rv.slot * (SLOT16 >> 4));
                        const bool half = has_fresh && q >= items - MT;  // at most 64 nodes
                        const uint32_t acc = q >= 2;
                        if (on) {
#pragma unroll
                            for (int kk = 0; kk < 8; ++kk)  // 16 tokens: 8 columns of P, two 8-token groups of V
                                if (kk < 4 || !half)
                                    mma_bf16_ts(tmem + O_COL + (uint32_t)(w * DH), tmem + (uint32_t)(w * 128 + kk * 8),
                                                dv + (uint64_t)(kk * (2 * GROUP_STRIDE >> 4)), idesc_o, kk > 0 ? 1u : acc);
                            if (MT == 1 || w) mma_commit(&ve[rv.slot]);
                            if (q == items - 1) mma_commit(&bars->pv_done);
                        }
                        __syncwarp();
                        if (MT == 1 || w) rv.next();
                    }
                    if (q + 2 < items) issue_s(q + 2, q + 3 == items, has_fresh && q + 2 >= items - MT);
                }
            }
            if (on) mma_commit(&bars->fin);  // completes when every MMA is done
            __syncwarp();
        }
    }
    // every MMA must be finished before TMEM and shared memory go away
    mbar_wait_drain(&bars->fin, 0);
    tc_fence_before();
    __syncthreads();
    // The next kernel may start only now, and the merge lets none start: blocks that waited on
    // SMs whose share was done slowed the others (200 sequences of 50 to 600 tokens: 104 -> 119 us).
    pdl_trigger();
    if (threadIdx.x == 0 && *abort && a.status) atomicOr(a.status, SP_DEV_TIMEOUT);
    if (warp == MMA) tmem_dealloc(tmem, 512);
}

// Merge of the pairs that lie in several shares (at most one starts in each share): a warp
// per (share, kv head, row), four dims a lane, the partials in share order, MERGE_AT of them
// under way together.  The kernel is all latency: with four at a time and two rows a warp, one
// sequence of 2048 tokens took 20.0 instead of 15.9 us.
constexpr int MERGE_THREADS = 128, MERGE_ROWS = 4, MERGE_AT = 8;
__global__ void __launch_bounds__(MERGE_THREADS) tree_tc_merge_kernel(const __grid_constant__ TreeArgs a, const int2 *split_tab) {
    pdl_wait();
    const int hv = blockIdx.x, j0 = blockIdx.y, Hv = a.Hkv * a.n_rb, g = hv / a.n_rb, rb = hv - g * a.n_rb;
    const int2 tab = __ldcg(split_tab + j0);
    if (tab.y <= 1) return;
    const int b = tab.x, nodes = a.n_nodes ? __ldg(a.n_nodes + b) : a.N;
    static_assert(MERGE_ROWS == MERGE_THREADS / 32, "a row a warp");
    const int lane = threadIdx.x & 31, c = lane * 4, n = checked_nodes(a, nodes, nullptr);
    const int q = blockIdx.z * MERGE_ROWS + (threadIdx.x >> 5), rr = rb * a.rb_rows + q;
    if (q < a.rb_rows && rr < a.R) {
        float m = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int e0 = 0; e0 < tab.y; e0 += MERGE_AT) {
            float2 ml[MERGE_AT];
            float4 ov[MERGE_AT];
#pragma unroll
            for (int e = 0; e < MERGE_AT; ++e) {
                const bool in = e0 + e < tab.y;
                const size_t slot = ((size_t)(j0 + e0 + e) * 2 + (e0 + e == 0)) * Hv + hv, row = slot * a.rb_rows + q;
                ml[e] = in ? __ldcg((const float2 *)(a.part_ml + row * 2)) : make_float2(-INFINITY, 0.f);
                ov[e] = in ? __ldcg((const float4 *)(a.part_o + row * DH + c)) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            float mn = m;
#pragma unroll
            for (int e = 0; e < MERGE_AT; ++e) mn = fmaxf(mn, ml[e].x);
            if (mn == -INFINITY) continue;
            const float al = m == -INFINITY ? 0.f : fmaxf(exp2f(m - mn), kLeastWeight);
            l *= al;
            o.x *= al, o.y *= al, o.z *= al, o.w *= al;
#pragma unroll
            for (int e = 0; e < MERGE_AT; ++e) {
                if (ml[e].x == -INFINITY) continue;
                const float w = fmaxf(exp2f(ml[e].x - mn), kLeastWeight);
                l += w * ml[e].y;
                o.x += w * ov[e].x, o.y += w * ov[e].y, o.z += w * ov[e].z, o.w += w * ov[e].w;
            }
            m = mn;
        }
        const int node = rr / a.G;
        const bool on = node < n && l != 0.f;
        const float s = on ? 1.f / l : 0.f;
        *(uint2 *)((bf16 *)a.out + ((size_t)b * a.N + node) * a.Hq * DH + (size_t)(g * a.G + rr - node * a.G) * DH + c) =
            on ? make_uint2(pack_bf16(o.x * s, o.y * s), pack_bf16(o.z * s, o.w * s)) : make_uint2(0, 0);
        if (a.lse && lane == 0) store_lse(a, b, node, g * a.G + rr - node * a.G, m, on ? l : 0.f);
    }
}

bool make_layout(const TreeArgs &a, bool e4, int mt, Layout *lay) {
    const int tab = (4 * a.B + 1) * 4;
    lay->off_tab = OFF_FRONT;
    lay->off_q = (OFF_FRONT + tab + 1023) & ~1023;
    int at = lay->off_q + mt * Q_TILE;
    lay->off_c = at;
    if (e4) at += CONV * (SLOT16 + PARAMS);
    lay->off_st = at;
    at += 2 * 8192;
    lay->off_sc = at;
    if (e4) at += MAX_AHEAD * 2 * TILE * 4;
    at = (at + 1023) & ~1023;
    const int slot = e4 ? SLOT8 : SLOT16, slots = (SMEM_MAX - 1024 - at) / slot;
    if (slots < 2) return false;
    // (8-bit: V's part is what the converters copy ahead)
    lay->nv = e4 ? (slots / 2 < MAX_AHEAD ? slots / 2 : MAX_AHEAD) : slots / 2 < MAX_RING ? slots / 2 : MAX_RING;
    lay->nk = slots - lay->nv < MAX_RING ? slots - lay->nv : MAX_RING;
    lay->off_k = at;
    lay->off_v = lay->off_k + lay->nk * slot;
    lay->smem = lay->off_v + lay->nv * slot + 1024;
    return lay->smem <= SMEM_MAX;
}

int row_tiles(const TreeArgs &a) { return a.rb_rows > 128 ? 2 : 1; }

template <bool E4, int TPC, int MT>
cudaError_t run(const TreeArgs &a, const Layout &lay, const CUtensorMap &mk, const CUtensorMap &mv, int2 *tab,
                cudaStream_t st) {
    static bool known[MAX_DEVICES] = {};
    const cudaError_t e = allow_smem(tree_tc_kernel<E4, TPC, MT>, SMEM_MAX, known);
    if (e != cudaSuccess) return e;
    return launch_k(tree_tc_kernel<E4, TPC, MT>, dim3(a.plan.tc_ctas), dim3(THREADS), (size_t)lay.smem, st, mk, mv, a,
                    lay, tab);
}

}  // namespace

bool tree_tc_supported(const TreeArgs &a) {
    Layout lay;
    return a.dh == DH && a.dtype == SP_BF16 && (a.cache.dtype == SP_BF16 || a.cache.dtype == SP_E4M3) && a.B <= MAX_B &&
           make_layout(a, a.cache.dtype == SP_E4M3, 2, &lay) &&
           (a.cache.kv.layout == SP_KV_CONTIGUOUS || (long long)a.cache.kv.n_pages * a.Hkv * a.cache.kv.page_size <= 0x7fffffffLL);
}

void plan_tree_tc(TreeArgs *a, int n_sm) {
    a->n_rb = ceil_div(a->R, 256);
    a->rb_rows = a->n_rb == 1 ? a->R : (ceil_div(a->R, a->n_rb) + 7) / 8 * 8;
    const int Hv = a->Hkv * a->n_rb;
    // (the tile list's numbers stay below 2^30)
    a->most_len = (int)min((long long)a->most_len, (long long)((1 << 30) / a->B - 1) * TILE);
    AttnArgs &p = a->plan;
    p.B = a->B;
    p.tc_ctas = attn_tc_ctas(n_sm, Hv);
    if (p.tc_ctas / Hv > MAX_GRP) p.tc_ctas = MAX_GRP * Hv;
    p.tc_min_tiles = kTreeMinTiles;
    p.tc_seg_cost = kTreeSegCost;
    p.tc_merge_kernel = 1;
}

int tree_tc_groups(const TreeArgs &a) { return a.plan.tc_ctas / (a.Hkv * a.n_rb); }
size_t tree_tc_slots(const TreeArgs &a) { return 2 * (size_t)a.plan.tc_ctas; }

cudaError_t launch_tree_tc(const TreeArgs &a, int2 *split_tab, cudaStream_t st) {
    const bool e4 = a.cache.dtype == SP_E4M3;
    const int mt = row_tiles(a);
    Layout lay;
    if (!make_layout(a, e4, mt, &lay)) return cudaErrorInvalidValue;
    CUtensorMap mk, mv;
    memset(&mk, 0, sizeof mk);
    memset(&mv, 0, sizeof mv);
    if (a.cache.kv.layout == SP_KV_PAGED) {
        const long long blocks = (long long)a.cache.kv.n_pages * a.Hkv;
        const int P = a.cache.kv.page_size;
        const bool ok = e4 ? encode_rows_u8(&mk, a.cache.kv.k_pool, blocks * P, P)
                           : encode_kv_pages_bf16(&mk, a.cache.kv.k_pool, blocks, P) &&
                                 encode_kv_pages_bf16(&mv, a.cache.kv.v_pool, blocks, P);
        if (!ok) return cudaErrorInvalidValue;
    }
    cudaError_t e;
    // Two M tiles against two blocks of up to 128 rows, which read the cache twice but overlap
    // scores and softmax: 8 sequences of 32768 tokens, 160 rows, 8-bit 389 against 432 us, bf16
    // 247 against 270; 32 of 500 to 9000, 200 rows, 296 against 321 and 199 against 199.  (One
    // sequence of 30000 tokens, whose cache the L2 holds: 66 against 56.)
    // Four copies of up to 32 rows against two and one: 128 sequences of 300 to 4000 tokens,
    // 4 rows, 8-bit, 197, 206, 263 us; 64 of 1024 to 8192, 32 rows, bf16 185, 189, 190, 8-bit
    // 198, 190, 233.  Two of up to 64 rows against one: 64 rows, bf16 190 and 192, 8-bit 223
    // and 253.
    if (mt == 2)
        e = e4 ? run<true, 128, 2>(a, lay, mk, mv, split_tab, st) : run<false, 128, 2>(a, lay, mk, mv, split_tab, st);
    else if (a.rb_rows <= 32)
        e = e4 ? run<true, 32, 1>(a, lay, mk, mv, split_tab, st) : run<false, 32, 1>(a, lay, mk, mv, split_tab, st);
    else if (a.rb_rows <= 64)
        e = e4 ? run<true, 64, 1>(a, lay, mk, mv, split_tab, st) : run<false, 64, 1>(a, lay, mk, mv, split_tab, st);
    else
        e = e4 ? run<true, 128, 1>(a, lay, mk, mv, split_tab, st) : run<false, 128, 1>(a, lay, mk, mv, split_tab, st);
    if (e != cudaSuccess) return e;
    return launch_k(tree_tc_merge_kernel, dim3(a.Hkv * a.n_rb, tree_tc_groups(a), ceil_div(a.rb_rows, MERGE_ROWS)), dim3(MERGE_THREADS), 0, st, a,
                    (const int2 *)split_tab);
}

}  // namespace sp

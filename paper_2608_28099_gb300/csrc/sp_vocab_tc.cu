// The vocabulary loss's products on tcgen05 tensor cores, bf16 with fp32 sums:
//   LOSS  logits of the kept tokens, whose epilogue leaves each row's (max, sum) over half a tile's columns
//   GRAD  the same logits, whose epilogue leaves g = dloss (p - 1_t) in bf16 for a piece of the vocabulary
//   DH    dh (+)= g W over the piece, fp32 planes
//   DW    dW = g^T h of the piece, bf16 (DW_LONG: from many tokens)
// Work: tiles of 256 x 256 (DH, DW) or 256 x tn (LOSS, GRAD: 64 to 256 rows of the vocabulary, VocabArgs::tn) by
// pairs of CTAs (tcgen05.mma.cta_group::2, M = 256: each CTA holds 128 rows of A and half of B's), K in blocks of 64 through a ring of TMA tiles, two accumulators in
// TMEM so that the epilogue of one tile runs beside the products of the next; persistent, a pair
// takes tiles in turn.  The operands lie as their tensors do: K contiguous (K-major) for the logits
// and for g in DH, the other index contiguous (MN-major) for W in DH and for both in DW; no
// operand is transposed in memory.  The number of kept tokens is read on the device: ignored tokens
// cost no product.
//
// What bounds it: the tensor pipe, and under it the board's power.  4096 tokens of 4096 (2744 kept)
// against 65536 rows: LOSS issues its MMAs back to back (1.22 M cycles, 1.21 M of them MMAs) and takes 720 us
// alone, 860 to 896 in a stream of calls on several boards, whose clocks settle near 1.65 GHz (1.64 to 1.71 PFLOP/s; a
// library product of such a stream 1.73).  GRAD takes 775 us alone, DH 780 to 800 in three splits (950 in one: 176 tiles for 76 pairs),
// DW of 2051 tokens of 2560 and 50021 rows 284.  The MMAs are issued by a whole warp in uniform registers, ring
// slots counted, not divided: by one thread that divided, LOSS took 870 us alone.  256 x 256 tiles by pairs load
// 64 bytes a cycle and SM from L2; seven stages instead of six change nothing.  Few tokens are bound by W:
// 48 tokens of 2560 against 32000 rows 33.4 to 34.4 us, 4.8 TB/s, of which 3 are the joining kernel and its launch.
#include <string.h>

#include "sp_gemm.cuh"
#include "sp_sm100.cuh"
#include "sp_train.cuh"

namespace sp {

namespace {

using namespace sm100;

enum { LOSS = 0, GRAD = 1, DH = 2, DW = 3, DW_LONG = 4 };
template <int KIND>
constexpr bool IS_DW = KIND == DW || KIND == DW_LONG;
template <int KIND>
constexpr bool IS_LOGITS = KIND == LOSS || KIND == GRAD;
constexpr float LOG2E = 1.4426950408889634f;
constexpr int TM = 256, TN = 256, BK = 64;       // a pair's tile; a CTA holds 128 x 256 of it.  LOSS and GRAD may take
                                                 // tiles of fewer columns (VocabArgs::tn)
constexpr int HALF = 128 * BK * 2;               // a CTA's part of an operand's k-block, 16 KB
constexpr int STAGE = 2 * HALF, STAGES = 6;
constexpr int OFF_BAR = STAGES * STAGE, OFF_OUT = OFF_BAR + 256;
constexpr int OUT_ROW = 64 + 16;                 // 32 bf16 of a row on their way out, padded
template <int KIND>
constexpr int SMEM = OFF_OUT + (KIND >= 2 ? 8 * 32 * OUT_ROW : 0) + 1024 /*align*/;
constexpr int THREADS = 352;                     // warps 0-7 epilogue, 8 TMA, 9 MMA (rank 0), 10 TMEM
constexpr int EPI_WARPS = 8, EPI_THREADS = 32 * EPI_WARPS, TMA = 8, MMA = 9, TMEM = 10;
constexpr int TMEM_COLS = 2 * TN;
// LOSS and GRAD add their logits up over 1024 of K at a time: the tensor core cuts what falls below an
// accumulator's 24 bits, which over longer sums shows in the loss (of its norm, with the whole of K in
// one accumulator: 2.0e-6 at d = 2560, 2.7e-6 at 4096, 4.5e-6 at 8192; so: 0.9e-6).  GRAD's logits are LOSS's, sum
// for sum, whatever the tiles' width: exp(l - lse) - 1 of a token that is almost sure of its target is as good as
// l and the log sum's logits agree (with the whole of K in one accumulator p - 1 of targets with logits of 30 was
// off by 3.6e-4 at d = 4096 and 9.4e-4 at 8192; so: by the log sum's own rounding, 1e-6).
// DW_LONG, the head's gradient from more than LONG_DW tokens, adds up that many at a time: in one accumulator that of
// 4000000 equal tokens was off by 2.6e-2.
constexpr int LONG_DW = 16384;
template <int KIND>
constexpr int ACC_KB = IS_LOGITS<KIND> ? 1024 / BK : KIND == DW_LONG ? LONG_DW / BK : 1 << 30;  // k-blocks of an accumulator

struct Ring {
    int slot = 0;
    uint32_t ph = 0;
    __device__ __forceinline__ void next() {
        if (++slot == STAGES) {
            slot = 0;
            ph ^= 1;
        }
    }
};
constexpr long long GRAD_BYTES = 512ll << 20;    // most bytes of a piece's g

template <int KIND>
struct Kind {
    static constexpr bool A_MN = IS_DW<KIND>, B_MN = KIND == DH || IS_DW<KIND>;
};

// Tiles of a product over `count` kept tokens and `piece` vocabulary rows.
struct Tiles {
    int m, n, kb, splits, per;
    __device__ __forceinline__ int items() const { return m * n * splits; }
};
template <int KIND>
__device__ __forceinline__ int count_of(const VocabArgs &a) {
    return KIND == LOSS && a.direct ? a.n : a.count->kept;
}
template <int KIND>
__device__ __forceinline__ int cols_of(const VocabArgs &a) {
    return IS_LOGITS<KIND> ? a.tn : TN;
}
template <int KIND>
__device__ __forceinline__ Tiles tiles_of(const VocabArgs &a, int count, int piece) {
    Tiles t;
    // (without a token one tile is formed whose rows are nobody's; DW's k-block 0 of g and h is cleared)
    t.m = IS_DW<KIND> ? ceil_div(piece, TM) : ceil_div(max(count, 1), TM);
    t.n = ceil_div(IS_LOGITS<KIND> ? piece : a.d, cols_of<KIND>(a));
    t.kb = KIND == DH ? ceil_div(piece, BK) : IS_DW<KIND> ? ceil_div(max(count, 1), BK) : ceil_div(a.d, BK);
    t.splits = 1, t.per = t.kb;
    if (KIND == DH) {
        const DhPlan p = *a.count;
        t.splits = p.splits, t.per = p.per;
    }
    return t;
}
struct Item {
    int m0, n0, nt, kb0, nkb, split;
};
// Neighbouring pairs take tiles that share what does not stay in L2: rows of the vocabulary (LOSS,
// GRAD), columns of W (DH); DW walks all of h's columns (which stay) for a tile of g.
template <int KIND>
__device__ __forceinline__ Item item_of(const Tiles &t, int it, int tn) {
    Item x;
    int m, n;
    if (IS_DW<KIND>) {
        n = it % t.n, m = it / t.n;
        x.split = 0;
    } else {
        m = it % t.m;
        const int q = it / t.m;
        n = q % t.n, x.split = q / t.n;
    }
    x.m0 = m * TM, x.n0 = n * tn, x.nt = n;
    x.kb0 = x.split * t.per;
    x.nkb = min(t.per, t.kb - x.kb0);  // (<= 0: a split that the last, shorter piece leaves nothing)
    return x;
}

template <int KIND>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
    vocab_tc_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                    const __grid_constant__ VocabArgs a, int v0) {
    typedef Kind<KIND> Ki;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t *full = (uint64_t *)(smem + OFF_BAR);  // rank 0's: both CTAs' copies
    uint64_t *empty = full + STAGES;
    uint64_t *acc_full = empty + STAGES;            // [2]
    uint64_t *acc_empty = acc_full + 2;             // [2], rank 0's: one arrival a CTA
    uint64_t *fin = acc_empty + 2;
    uint32_t *tmem_slot = (uint32_t *)(fin + 1);
    volatile int *abort = (volatile int *)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int cl = blockIdx.x >> 1, n_cl = gridDim.x >> 1;

    if (warp == TMA && lane == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&acc_full[i], 1);
            mbar_init(&acc_empty[i], 2);
        }
        mbar_init(fin, 1);
        *abort = 0;
        fence_mbar_init();
        prefetch_tmap(&map_a);
        prefetch_tmap(&map_b);
    }
    __syncwarp();
    cluster_arrive();  // both CTAs' barriers exist before either signals the other's
    if (warp == TMEM) tmem_alloc_pair(tmem_slot, TMEM_COLS);
    cluster_wait();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const int piece = min(a.piece, a.V - v0);
    const int tn = cols_of<KIND>(a);              // (a CTA holds half of B's rows)
    // both CTAs' bytes; the logits of up to 128 tokens leave A's other rows as they are (nobody's rows of D)
    const bool short_a = IS_LOGITS<KIND> && a.box < 128;
    const uint32_t stage_tx = (short_a ? (uint32_t)a.box * BK * 2 : 2 * HALF) + (uint32_t)tn * BK * 2;

    if (warp == TMA && lane == 0) {
        // what is read again soon stays in L2, the vocabulary's rows of LOSS pass through
        const uint64_t pol_a = IS_LOGITS<KIND> ? policy_evict_last() : policy_evict_normal();
        const uint64_t pol_b = KIND == LOSS ? policy_evict_first() : IS_DW<KIND> ? policy_evict_last() : policy_evict_normal();
        // Up to 256 tokens the first tile of GRAD is known before they are counted, and W does not depend
        // on them: its k-blocks are asked for while the kernel in front still runs (which has
        // waited for the caller's earlier work before it let this one start).
        int pre = 0;
        if (KIND == GRAD && a.pad == TM && cl < ceil_div(piece, tn)) {
            pre = min(STAGES, ceil_div(a.d, BK));
            for (int i = 0; i < pre; ++i) {
                if (rank == 0) mbar_arrive_expect_tx(&full[i], stage_tx);
                tma_load_2d_pair(smem + i * STAGE + HALF, &map_b, map_rank(&full[i], 0), i * BK, v0 + cl * tn + (int)rank * (tn / 2), pol_b);
            }
        }
        pdl_wait();
        const Tiles t = tiles_of<KIND>(a, count_of<KIND>(a), piece);
        const int n_items = t.items();
        Ring rg;
        int filled = 0;
        bool ok = true;
        for (int it = cl; ok && it < n_items; it += n_cl) {
            const Item x = item_of<KIND>(t, it, tn);
            const int ma = x.m0 + (int)rank * 128, nb = x.n0 + (int)rank * (tn / 2);
            for (int i = 0; i < x.nkb; ++i, rg.next(), ++filled) {
                const int s = rg.slot, k = (x.kb0 + i) * BK;
                // (a stage asked for in front is free, and may be read already where the other CTA had all else of
                // it: its barrier's phase is then one ahead, and the first one would be waited for in vain)
                if (filled >= pre && !mbar_wait(&empty[s], rg.ph ^ 1, abort)) {
                    ok = false;
                    break;
                }
                if (rank == 0 && filled >= pre) mbar_arrive_expect_tx(&full[s], stage_tx);
                const uint32_t bar = map_rank(&full[s], 0);
                uint8_t *sa = smem + s * STAGE, *sb = sa + HALF;
                if (Ki::A_MN) {
                    tma_load_2d_pair(sa, &map_a, bar, ma, k, pol_a);
                    tma_load_2d_pair(sa + HALF / 2, &map_a, bar, ma + 64, k, pol_a);
                } else if (!short_a || rank == 0) {
                    tma_load_2d_pair(sa, &map_a, bar, k, ma, pol_a);
                }
                if (Ki::B_MN) {
                    const int kv = KIND == DH ? v0 + k : k;
                    tma_load_2d_pair(sb, &map_b, bar, nb, kv, pol_b);
                    tma_load_2d_pair(sb + HALF / 2, &map_b, bar, nb + 64, kv, pol_b);
                } else if (filled >= pre) {
                    tma_load_2d_pair(sb, &map_b, bar, k, v0 + nb, pol_b);
                }
            }
        }
        // nothing may land in this CTA after it is gone: the last use of every stage has been read
        for (int j = 0; j < STAGES; ++j, rg.next())
            if (!mbar_wait_drain(&empty[rg.slot], rg.ph ^ 1)) break;
    } else if (warp == MMA && rank == 0) {
        // by the whole warp, the instructions under `on` (see elect_one)
        const bool on = elect_one();
        const uint32_t idesc = idesc_bf16_f32(TM, tn) | (Ki::A_MN ? 1u << 15 : 0u) | (Ki::B_MN ? 1u << 16 : 0u);
        // a step of 16 along K: 32 bytes of a K-major row, 16 rows of 128 bytes of an MN-major tile
        constexpr uint64_t step_a = Ki::A_MN ? 2048 >> 4 : 32 >> 4, step_b = Ki::B_MN ? 2048 >> 4 : 32 >> 4;
        const uint64_t da0 = Ki::A_MN ? sw128_mnmajor_desc(smem, HALF / 2) : sw128_kmajor_desc(smem);
        const uint64_t db0 = Ki::B_MN ? sw128_mnmajor_desc(smem + HALF, HALF / 2) : sw128_kmajor_desc(smem + HALF);
        pdl_wait();
        const Tiles t = tiles_of<KIND>(a, count_of<KIND>(a), piece);
        const int n_items = t.items();
        Ring rg;
        int n = 0;  // accumulators
        bool ok = true;
#pragma unroll 1
        for (int it = cl; ok && it < n_items; it += n_cl) {
            const Item x = item_of<KIND>(t, it, tn);
#pragma unroll 1
            for (int i0 = 0; ok && i0 < x.nkb; i0 += ACC_KB<KIND>) {
                const int buf = n & 1, end = min(ACC_KB<KIND>, x.nkb - i0);
                const uint32_t acc = tmem + (uint32_t)(buf * TN);
                // both CTAs' epilogues have read what this accumulator held
                if (n >= 2) ok = __all_sync(0xffffffffu, mbar_wait_cluster(&acc_empty[buf], ((n >> 1) - 1) & 1, abort));
                ++n;
#pragma unroll 1
                for (int i = 0; i < end; ++i, rg.next()) {
                    ok = ok && mbar_wait_warp(&full[rg.slot], rg.ph, abort);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t da = da0 + (uint32_t)(rg.slot * (STAGE >> 4)), db = db0 + (uint32_t)(rg.slot * (STAGE >> 4));
                    if (on) {
#pragma unroll
                        for (int kk = 0; kk < BK / 16; ++kk)
                            mma_bf16_pair(acc, da + step_a * kk, db + step_b * kk, idesc, i > 0 || kk > 0 ? 1u : 0u);
                        mma_commit_pair(&empty[rg.slot]);
                        if (i == end - 1) mma_commit_pair(&acc_full[buf]);
                    }
                    __syncwarp();
                }
            }
        }
        if (on) mma_commit_pair(fin);  // every MMA is finished before TMEM and shared memory go away
        __syncwarp();
        mbar_wait_drain(fin, 0);
    } else if (warp < EPI_WARPS) {
        // a row a thread: warp w reads TMEM lanes 32 (w & 3).. and columns 128 (w >> 2)..
        const int quad = warp & 3, half = warp >> 2, row = quad * 32 + lane;
        pdl_wait();
        const int count = count_of<KIND>(a);
        const Tiles t = tiles_of<KIND>(a, count, piece);
        const int n_items = t.items();
        int n = 0;  // accumulators read
        const auto wait_acc = [&]() {
            const bool have = __all_sync(0xffffffffu, mbar_wait(&acc_full[n & 1], (n >> 1) & 1, abort));
            tc_fence_after();
            return have;
        };
        const auto acc_at = [&]() { return tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)((n & 1) * TN + half * (tn / 2)); };
        // All epilogue warps meet here, whatever their waits said, and learn of the others': one that had left
        // would be waited for without a limit.  (Arrivals of each warp for itself: 40000 tokens of 512 against 2000 rows 147
        // instead of 140 us.)
        const auto release_acc = [&](bool have) {
            int all;
            tc_fence_before();
            asm volatile(
                "{\n\t.reg .pred p, q;\n\t"
                "setp.ne.s32 q, %1, 0;\n\t"
                "barrier.cta.red.and.pred p, 1, %2, q;\n\t"
                "selp.s32 %0, 1, 0, p;\n\t}"
                : "=r"(all)
                : "r"((int)have), "n"(EPI_THREADS)
                : "memory");
            if (all && threadIdx.x == 0) mbar_arrive_remote(map_rank(&acc_empty[n & 1], 0));
            ++n;
            return all != 0;
        };
        // bf16 rows go out through shared memory, 64 bytes of a row by four lanes: where a lane's four rows start (own:
        // where this one's does, or -1), and 32 columns of every lane's row
        uint8_t *stage = smem + OFF_OUT + warp * 32 * OUT_ROW;
        const auto rows_of = [&](long long own, long long (&out_row)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) out_row[i] = __shfl_sync(0xffffffffu, own, i * 8 + (lane >> 2));
        };
        const auto rows_out = [&](const float (&v)[32], bf16 *out, const long long (&out_row)[4], int col) {
            __syncwarp();  // (the columns before are read)
#pragma unroll
            for (int j = 0; j < 32; j += 8)
                *(uint4 *)(stage + lane * OUT_ROW + j * 2) = make_uint4(pack2_bf16(v[j], v[j + 1]), pack2_bf16(v[j + 2], v[j + 3]),
                                                                        pack2_bf16(v[j + 4], v[j + 5]), pack2_bf16(v[j + 6], v[j + 7]));
            __syncwarp();
            col += (lane & 3) * 8;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (out_row[i] >= 0 && col < a.d)
                    *(uint4 *)(out + out_row[i] + col) = *(const uint4 *)(stage + (i * 8 + (lane >> 2)) * OUT_ROW + (lane & 3) * 16);
        };
        bool ok = true;
        for (int it = cl; ok && it < n_items; it += n_cl) {
            const Item x = item_of<KIND>(t, it, tn);
            if (KIND == DH && x.nkb <= 0) continue;
            const int m = x.m0 + (int)rank * 128 + row, c0 = x.n0 + half * (tn / 2);  // row, first column
            VocabRow info{0.f, 0.f, -1, 0};
            if (KIND == LOSS && a.direct) {
                const int target = m < count ? a.targets[m] : -1;
                if (has_target(target, a.V)) info.target = target;
                else if (target >= a.V && it == 0 && a.status) atomicOr(a.status, SP_DEV_BAD_ROW);
            } else if (IS_LOGITS<KIND> && m < count) {
                info = a.rows[m];
            }
            if constexpr (IS_LOGITS<KIND> || KIND == DW_LONG) {
                constexpr int CH = 16;  // columns read at a time; those behind the half's last one are not looked at
                float v[TN / 2];
#pragma unroll
                for (int c = 0; c < TN / 2; ++c) v[c] = 0.f;
#pragma unroll 1
                for (int k = 0; k < x.nkb; k += ACC_KB<KIND>) {
                    ok = wait_acc();
                    const uint32_t at = acc_at();
#pragma unroll
                    for (int c = 0; c < TN / 2; c += CH) {
                        if (c >= tn / 2) break;
                        float u[CH];
                        tmem_ld16(at + c, u);
#pragma unroll
                        for (int j = 0; j < CH; ++j) v[c + j] += u[j];
                    }
                    ok = release_acc(ok);
                    if (!ok) break;
                }
                if (!ok) break;
                if constexpr (KIND == GRAD) {
                    const int left = m < count ? piece - c0 : 0, hit = info.target - v0 - c0;
                    uint4 *to = (uint4 *)((bf16 *)a.grad + (size_t)m * a.piece + c0);
#pragma unroll
                    for (int c = 0; c < TN / 2; c += 32) {  // (64 bytes of a row together)
                        if (c >= tn / 2) break;
                        uint32_t w[16];
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            float g[2];
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const float p = fast_exp2((v[c + j + q] - info.lse) * LOG2E);
                                g[q] = c + j + q < left ? (c + j + q == hit ? p - 1.f : p) * info.g : 0.f;
                            }
                            w[j / 2] = pack2_bf16(g[0], g[1]);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) to[c / 8 + j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
                    }
                    continue;
                }
                if constexpr (KIND == DW_LONG) {
                    long long out_row[4];
                    rows_of(m < piece ? (long long)(v0 + m) * a.ws : -1, out_row);
#pragma unroll
                    for (int c = 0; c < TN / 2; c += 32) {
                        float u[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) u[j] = v[c + j];
                        rows_out(u, (bf16 *)a.dw, out_row, c0 + c);
                    }
                    continue;
                }
                const int left = min(piece - c0, tn / 2), hit = info.target - c0;
                float mx = -INFINITY, z = 0.f;
#pragma unroll
                for (int c = 0; c < TN / 2; ++c) {
                    if (c >= left) v[c] = -INFINITY;
                    mx = fmaxf(mx, v[c]);
                }
                if (hit >= 0 && hit < left) {  // (once a row)
#pragma unroll
                    for (int c = 0; c < TN / 2; ++c) z = c == hit ? v[c] : z;
                    a.at[m] = z;
                }
                const float mu = mx == -INFINITY ? 0.f : mx;
                float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < TN / 2; ++c) s4[c & 3] += fast_exp2((v[c] - mu) * LOG2E);
                if (m < count) a.part[(size_t)m * a.parts + 2 * x.nt + half] = make_float2(mx, (s4[0] + s4[1]) + (s4[2] + s4[3]));
            } else {
                // bf16 rows: dW's, and dh's where it belongs if it comes in one part
                const bool rows = KIND == DW || (KIND == DH && t.splits == 1 && a.n_pieces == 1);
                bf16 *const out = KIND == DW ? (bf16 *)a.dw : (bf16 *)a.dh;
                long long out_row[4];
                if (rows) {
                    long long own = -1;
                    if (KIND == DW && m < piece) own = (long long)(v0 + m) * a.ws;
                    if (KIND == DH && m < count) own = (long long)a.rows[m].token * a.hs;
                    rows_of(own, out_row);
                }
                ok = wait_acc();
                const uint32_t at = acc_at();
#pragma unroll 1
                for (int c = 0; c < TN / 2; c += 32) {
                    float v[32];
                    __syncwarp();  // (rows that store nothing have skipped ahead)
                    tmem_ld32(at + c, v);
                    if (rows) {
                        rows_out(v, out, out_row, c0 + c);
                    } else {
                        if (m >= count) continue;
                        float *to = a.acc + ((size_t)x.split * (t.m * TM) + m) * a.d + c0 + c;
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            if (c0 + c + j >= a.d) break;
                            float4 y = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                            if (v0) {
                                const float4 z = *(const float4 *)(to + j);
                                y.x += z.x, y.y += z.y, y.z += z.z, y.w += z.w;
                            }
                            *(float4 *)(to + j) = y;
                        }
                    }
                }
                ok = release_acc(ok);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    pdl_trigger();
    if (threadIdx.x == 0 && *abort && a.status) atomicOr(a.status, SP_DEV_TIMEOUT);
    // rank 0's last commit arrives on both CTAs' barriers: each waits until it has landed
    if (threadIdx.x == 0 && rank != 0) mbar_wait_drain(fin, 0);
    __syncwarp();
    cluster_sync();  // no signal or MMA of the other CTA may still target this one
    if (warp == TMEM) tmem_dealloc_pair(tmem, TMEM_COLS);
}

template <int KIND>
cudaError_t run(const VocabArgs &a, const CUtensorMap &ma, const CUtensorMap &mb, int v0, cudaStream_t st) {
    static bool known[MAX_DEVICES] = {};
    const cudaError_t e = allow_smem(vocab_tc_kernel<KIND>, SMEM<KIND>, known);
    if (e != cudaSuccess) return e;
    const int piece = a.V - v0 < a.piece ? a.V - v0 : a.piece;
    const long long m = IS_DW<KIND> ? ceil_div(piece, TM) : a.pad / TM;
    const long long n = ceil_div(IS_LOGITS<KIND> ? piece : a.d, IS_LOGITS<KIND> ? a.tn : TN);
    const long long items = m * n * (KIND == DH ? 16 : 1);
    const int pairs = a.pairs;
    return launch_k(vocab_tc_kernel<KIND>, dim3(2 * (items < pairs ? (unsigned)items : (unsigned)pairs)), dim3(THREADS), (size_t)SMEM<KIND>,
                    st, ma, mb, a, v0);
}

}  // namespace

bool vocab_tc_supported(const VocabArgs &a) {
    return a.dtype == SP_BF16 && a.d % 8 == 0 && a.hs % 8 == 0 && a.ws % 8 == 0;
}

void plan_vocab_tc(VocabArgs *a, bool backward, int n_sm) {
    a->tm = TM;
    a->pad = ceil_div(a->n, TM) * TM;
    a->pairs = n_sm / 2 > 0 ? n_sm / 2 : 1;
    a->tn = TN;
    a->box = a->n <= 128 ? ceil_div(a->n, 8) * 8 : 128;
    a->direct = !backward && a->n <= TM;
    // Tiles of the width whose rounds over the pairs read the fewest rows of W (48 tokens, 32000 rows: 2 x 224 instead
    // of 2 x 256 a pair), a tile's ends costing some 64 of them; g's in whole k-blocks of dh's product (6364 rows of
    // 4096, 48 tokens: 26 us with 256, 22 with 128; 67629 of 1888, 8 tokens: 57 and 64).
    long long least = 1ll << 62;
    for (int tn = TN; tn >= 64; tn -= backward ? 64 : 32) {
        const long long rows = ceil_div_ll((long long)ceil_div(a->V, tn) * (a->pad / TM), a->pairs) * (tn + 64);
        if (rows < least) least = rows, a->tn = tn;
    }
    const int tiles = ceil_div(a->V, a->tn);
    a->parts = 2 * tiles;
    a->piece = tiles * a->tn;
    a->n_pieces = 1;
    if (!backward) return;
    long long most = GRAD_BYTES / 2 / a->pad / a->tn;  // tiles of a piece
    if (most < 1) most = 1;
    a->n_pieces = (int)ceil_div_ll(tiles, most);
    a->piece = ceil_div(tiles, a->n_pieces) * a->tn;
    a->n_pieces = ceil_div(a->V, a->piece);
}

// (The maps of the kept tokens' rows end behind the n-th: rows of a tile that cannot be there are zeros that
// nothing fetches.  48 tokens against 32000 rows of 2560: 38 us with all 256 rows of the tile.)
cudaError_t launch_vocab_loss_tc(const VocabArgs &a, cudaStream_t st) {
    CUtensorMap mh, mw;
    if (!(a.direct ? encode_tile_bf16(&mh, a.h, a.d, a.n, a.hs, a.box) : encode_tile_bf16(&mh, a.hc, a.d, a.n, a.d, 128)) ||
        !encode_tile_bf16(&mw, a.w, a.d, a.V, a.ws, a.tn / 2))
        return cudaErrorInvalidValue;
    return run<LOSS>(a, mh, mw, 0, st);
}

cudaError_t launch_vocab_backward_tc(const VocabArgs &a, cudaStream_t st) {
    CUtensorMap mh, mw, mg, mwt, mgt, mht;
    if (!encode_tile_bf16(&mh, a.hc, a.d, a.n, a.d, a.box) || !encode_tile_bf16(&mw, a.w, a.d, a.V, a.ws, a.tn / 2) ||
        !encode_tile_bf16(&mg, a.grad, a.piece, a.pad, a.piece, 128) || !encode_tile_bf16(&mwt, a.w, a.d, a.V, a.ws, 64) ||
        !encode_tile_bf16(&mgt, a.grad, a.piece, a.pad, a.piece, 64) || !encode_tile_bf16(&mht, a.hc, a.d, a.n, a.d, 64))
        return cudaErrorInvalidValue;
    for (int i = 0; i < a.n_pieces; ++i) {
        const int v0 = i * a.piece;
        cudaError_t e = run<GRAD>(a, mh, mw, v0, st);
        if (e == cudaSuccess) e = run<DH>(a, mg, mwt, v0, st);
        if (e == cudaSuccess && a.dw) e = a.n > LONG_DW ? run<DW_LONG>(a, mgt, mht, v0, st) : run<DW>(a, mgt, mht, v0, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace sp

// Cross entropy of tokens over a large vocabulary from the hidden states, and its gradients (the
// readout of a draft layer's hidden states by a language model's head, Sec. 3.1 and the head ablation
// of Sec. 5), without keeping the logits l = h W^T:
//   lse = log sum_v exp l_v,   loss = lse - l_t
//   g_v = dloss (exp(l_v - lse) - [v = t]),   dh = g W,   dW = g^T h
// Here: what stands around the products (counting off the tokens that have a target, joining the
// parts of a row's sum, writing gradients back to their tokens), and the products on CUDA cores in
// fp32 for fp32 rows and unaligned ones.  The tensor-core products are in sp_vocab_tc.cu.
#include <type_traits>

#include "sp_train.cuh"

namespace sp {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int THREADS = 256, WARPS = THREADS / 32;

// The splits along the vocabulary of dh's tiles (tm rows a tile) for `kept` tokens: the fewest rounds of
// k-blocks over the machine's `pairs` units, a split's partial costing some itself (two passes over it: `plane`
// k-blocks a tile; a k-block of 256 x 256 x 64 takes a pair 0.27 us, in which two passes over 0.3 tiles of fp32
// partials fit the HBM's share of a pair; a block of CUDA cores some 0.7 us, which a partial does not weigh
// against).  By a warp, a number of splits a lane.
constexpr int MAX_SPLITS = 16;
__device__ __forceinline__ DhPlan plan_dh(const VocabArgs &a, int kept, int lane) {
    const int tm = a.tm, bk = a.tensor ? 64 : 2048 / tm, kb = ceil_div(min(a.piece, a.V), bk);
    const int m_tiles = ceil_div(max(kept, 1), tm), n_tiles = ceil_div(a.d, tm), s = lane + 1, per = ceil_div(kb, s);
    const float plane = a.tensor ? 24.f : 2.f;
    float cost = 3e38f;
    if ((long long)m_tiles * n_tiles < 8ll * a.pairs) {
        const int tiles = m_tiles * n_tiles;
        if (s <= MAX_SPLITS && tiles * lane < 8 * a.pairs && lane * per < kb)
            cost = (float)ceil_div(tiles * s, a.pairs) * (float)(per + 4) + (s > 1 ? plane * (float)(s * tiles) / (float)a.pairs : 0.f);
    } else if (lane == 0) {
        cost = 0.f;
    }
    float least = cost;
#pragma unroll
    for (int o = 16; o; o >>= 1) least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
    const int best = __ffs(__ballot_sync(0xffffffffu, cost == least));  // (the fewest splits of equal cost)
    return DhPlan{kept, m_tiles, best, __shfl_sync(0xffffffffu, per, best - 1)};
}

// Rows of the products: a token with a target gets the next row.  Every block counts the targets in
// front of its own `per` tokens and in all (n ints from L2), then copies its rows where they go,
// a warp a row, and clears what is known to be 0: losses and gradients of the others, and
// rows behind the last one up to a whole k-block.
template <typename T>
__global__ void __launch_bounds__(THREADS) vocab_keep_kernel(const __grid_constant__ VocabArgs a, int per, int backward) {
    __shared__ int front[WARPS], total[WARPS], here[WARPS], pos[THREADS];
    pdl_wait();
    pdl_trigger();
    const int t0 = blockIdx.x * per, t1 = min(a.n, t0 + per), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int f = 0, all = 0;
    bool bad = false;
#pragma unroll 8
    for (int t = threadIdx.x; t < a.n; t += THREADS) {
        const int v = a.targets[t];
        const bool on = has_target(v, a.V);
        bad |= v >= a.V;
        all += on;
        f += on && t < t0;
    }
    f = __reduce_add_sync(0xffffffffu, f);
    all = __reduce_add_sync(0xffffffffu, all);
    if (lane == 0) front[warp] = f, total[warp] = all;
    __syncthreads();
    f = all = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) f += front[w], all += total[w];
    if (blockIdx.x == 0) {
        if (bad && a.status) atomicOr(a.status, SP_DEV_BAD_ROW);
        if (warp == 0) {
            const DhPlan plan = backward ? plan_dh(a, all, lane) : DhPlan{all, 0, 0, 0};
            if (lane == 0) *a.count = plan;
        }
    }
    for (int g0 = t0; g0 < t1; g0 += THREADS) {  // 256 of its tokens at a time (most blocks have few)
        const int t = g0 + threadIdx.x, v = t < t1 ? a.targets[t] : -1;
        const bool on = has_target(v, a.V);
        const unsigned mask = __ballot_sync(0xffffffffu, on);
        __syncthreads();  // (the positions before are read)
        if (lane == 0) here[warp] = __popc(mask);
        __syncthreads();
        int p = f + __popc(mask & ((1u << lane) - 1));
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) p += here[w];
            f += here[w];
        }
        pos[threadIdx.x] = on ? p : -1;
        if (on) {
            VocabRow r{0.f, 0.f, v, t};
            if (backward) {
                r.lse = a.lse_in[t];
                r.g = a.dloss ? a.dloss[t] : 1.f;
            }
            a.rows[p] = r;
        } else if (t < t1 && !backward) {
            a.loss[t] = 0.f;
            a.lse[t] = 0.f;
        }
        __syncthreads();
        const int end = min(THREADS, t1 - g0);
        for (int i = warp; i < end; i += WARPS) {
            const int q = pos[i];
            if (q < 0) {
                if (backward)
                    for (int e = lane; e < a.d; e += 32) ((T *)a.dh)[(size_t)(g0 + i) * a.hs + e] = from_f<T>(0.f);
            } else if (!a.tensor) {
                const T *src = (const T *)a.h + (size_t)(g0 + i) * a.hs;
                T *dst = (T *)a.hc + (size_t)q * a.d;
#pragma unroll 8
                for (int e = lane; e < a.d; e += 32) dst[e] = src[e];
            } else {
                const uint4 *src = (const uint4 *)((const T *)a.h + (size_t)(g0 + i) * a.hs);
                uint4 *dst = (uint4 *)((bf16 *)a.hc + (size_t)q * a.d);  // (d is a multiple of 8, rows are aligned)
                constexpr int AT_ONCE = 8;
                for (int e0 = lane; e0 < a.d / 8; e0 += 32 * AT_ONCE) {
                    uint4 v4[AT_ONCE];
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k)
                        if (e0 + 32 * k < a.d / 8) v4[k] = src[e0 + 32 * k];
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k)
                        if (e0 + 32 * k < a.d / 8) dst[e0 + 32 * k] = v4[k];
                }
            }
        }
    }
    if (a.tensor && backward) {
        const int end = min(a.pad, max(ceil_div(all, 64), 1) * 64);
        for (int p = all + blockIdx.x; p < end; p += gridDim.x)
            for (int e = threadIdx.x; e < a.d / 8; e += THREADS) *(uint4 *)((bf16 *)a.hc + (size_t)p * a.d + e * 8) = make_uint4(0, 0, 0, 0);
    }
}

// Loss and log sum of a row from its parts, a warp a row, parts joined in a fixed order.
__global__ void __launch_bounds__(THREADS) vocab_finish_loss_kernel(const __grid_constant__ VocabArgs a) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, p = blockIdx.x * WARPS + (threadIdx.x >> 5);
    int token = p;
    if (a.direct) {
        if (p >= a.n) return;
        if (!has_target(a.targets[p], a.V)) {
            if (lane == 0) a.loss[p] = a.lse[p] = 0.f;
            return;
        }
    } else {
        if (p >= a.count->kept) return;
        token = a.rows[p].token;
    }
    const float2 *part = a.part + (size_t)p * a.parts;
    float m = -INFINITY, l = 0.f;
    constexpr int AT_ONCE = 8;
    for (int i0 = lane; i0 < a.parts; i0 += 32 * AT_ONCE) {
        float2 v[AT_ONCE];
        float mn = m;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) v[k] = i0 + 32 * k < a.parts ? part[i0 + 32 * k] : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) mn = fmaxf(mn, v[k].x);
        if (m != -INFINITY) l *= exp2f((m - mn) * LOG2E);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)  // (without a maximum: 0, or NaN)
            l += v[k].x == -INFINITY ? v[k].y : v[k].y * exp2f((v[k].x - mn) * LOG2E);
        m = mn;
    }
    float top = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    l = m == -INFINITY ? l : l * exp2f((m - top) * LOG2E);
#pragma unroll
    for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (lane == 0) {
        const float lg = logf(l);
        a.lse[token] = top + lg;
        a.loss[token] = (top - a.at[p]) + lg;  // (the maximum and the target's logit may be large and close)
    }
}

// dh of the kept tokens: the splits' parts added in order.
template <typename T>
__global__ void __launch_bounds__(THREADS) vocab_finish_dh_kernel(const __grid_constant__ VocabArgs a) {
    pdl_wait();
    pdl_trigger();
    const int p = blockIdx.x;
    const DhPlan plan = *a.count;
    if (p >= plan.kept || (a.tensor && plan.splits == 1 && a.n_pieces == 1)) return;  // (dh is written)
    T *to = (T *)a.dh + (size_t)a.rows[p].token * a.hs;
    const float *from = a.acc + (size_t)p * a.d;
    const size_t plane = (size_t)plan.m_tiles * a.tm * a.d;
    if (a.tensor) {  // (d a multiple of 8, rows aligned)
        for (int e = threadIdx.x * 4; e < a.d; e += THREADS * 4) {
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
            constexpr int AT_ONCE = 8;  // planes under way together
            for (int q0 = 0; q0 < plan.splits; q0 += AT_ONCE) {
                float4 v[AT_ONCE];
#pragma unroll
                for (int q = 0; q < AT_ONCE; ++q)
                    v[q] = q0 + q < plan.splits ? __ldcs((const float4 *)(from + (q0 + q) * plane + e)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int q = 0; q < AT_ONCE; ++q) s.x += v[q].x, s.y += v[q].y, s.z += v[q].z, s.w += v[q].w;
            }
            *(uint2 *)((bf16 *)to + e) = make_uint2(pack2_bf16(s.x, s.y), pack2_bf16(s.z, s.w));
        }
    } else {
        for (int e = threadIdx.x; e < a.d; e += THREADS) {
            float s = 0.f;
#pragma unroll 8
            for (int q = 0; q < plan.splits; ++q) s += from[q * plane + e];
            to[e] = from_f<T>(s);
        }
    }
}

// ---------------------------------------------------------------------------
// Products on CUDA cores: C[m][n] = sum_k A(m, k) B(n, k), the operands through two buffers in shared
// memory, the next ones' loads under way beside the products, fp32 throughout; dh's tiles split along K
// where they are few.  Tiles of 64 x 64 and 32 of K at a time, 4 x 4 elements a thread, or where these leave SMs
// idle (VocabArgs::tm) of 32 x 32 and 64 of K: a k-block of the first takes an SM 0.55 us of FMAs alone.
// There dh and dW go by 4 x 4, four groups of 64 threads adding up a quarter of K each; the logits by 2 x 2, so that
// they are the same sums, k after k, in every kernel: exp(l - lse) is only as good as the lse's logits and these agree
// (by quarters: errors of 4e-6 instead of 6e-7 of the gradients' norm with another kernel's lse).
enum { LOSS = 0, GRAD = 1, DH = 2, DW = 3 };

// dh and dW: products of this many of K are added up in one number, which then joins the sum of those in front with
// what that addition cuts off, so that sums over a large vocabulary or many tokens lose no more than short ones (in
// one number dW of 65536 equal tokens was off by 8e-4, of 4000000 by 4.5e-2, dh over 131072 equal rows by 2e-4).
constexpr int RUN = 512;

template <int BM>
struct Simt {
    static constexpr int BK = 2048 / BM, LOADS = BM * BK / THREADS;
    struct Smem {
        float a[2][BK][BM + 4], b[2][BK][BM + 4];
        VocabRow rows[BM];
    };
    struct BackSmem : Smem {
        float2 runs[16][THREADS];  // a thread's sums of runs, and what they cut off (in registers: one block an SM)
    };
};
// E x E elements a thread, a tile by GROUP threads.
template <int KIND, int BM>
struct Cut {
    static constexpr int E = BM == 32 && (KIND == LOSS || KIND == GRAD) ? 2 : 4;
    static constexpr int PER_ROW = BM / E, GROUP = PER_ROW * PER_ROW, GROUPS = THREADS / GROUP;
};

template <typename T, int KIND>
struct SimtA {
    typedef typename std::conditional<KIND == LOSS || KIND == GRAD, T, float>::type type;
};
template <typename T, int KIND, int BM>
__device__ __forceinline__ void simt_tile(const VocabArgs &a, int v0, int n0, int m0, int split, typename Simt<BM>::Smem &s,
                                          float2 (*runs)[THREADS] = nullptr) {
    typedef Simt<BM> S;
    typedef Cut<KIND, BM> C;
    constexpr int BK = S::BK, LOADS = S::LOADS, GROUPS = C::GROUPS, E = C::E;
    const DhPlan plan = *a.count;
    const int count = plan.kept;
    const int piece = min(a.piece, a.V - v0);
    // M, N, K of this product
    const int M = KIND == DW ? piece : count, N = KIND == LOSS || KIND == GRAD ? piece : a.d;
    const int K = KIND == DH ? piece : KIND == DW ? count : a.d;
    if (m0 >= M) return;
    int k_lo = 0, k_hi = K, plane_rows = 0;
    if (KIND == DH) {
        if (split >= plan.splits) return;
        k_lo = min(K, split * plan.per * BK);  // (the last piece may leave a split nothing: zeros)
        k_hi = min(K, k_lo + plan.per * BK);
        plane_rows = plan.m_tiles * BM;
    }
    const int tid = threadIdx.x, group = tid / C::GROUP, at = tid % C::GROUP;
    const int ty = at / C::PER_ROW, tx = at % C::PER_ROW;
    if (KIND != DW) {
        if (tid < BM) s.rows[tid] = m0 + tid < count ? a.rows[m0 + tid] : VocabRow{0.f, 0.f, -1, 0};
        __syncthreads();
    }
    // element (row, k) of the tile's A and B: at p[row * rows + k * steps]; neighbouring threads along whichever
    // index is contiguous in memory (k: 8 by 4 rows, whose places in shared memory lie in 32 banks)
    constexpr bool A_MN = KIND == DW, B_MN = KIND == DH || KIND == DW;
    typedef typename SimtA<T, KIND>::type TA;
    const TA *pa0;
    const T *pb0;
    size_t rows_a = 1, rows_b = 1, step_a = 1, step_b = 1;
    if constexpr (KIND == LOSS || KIND == GRAD) {
        pa0 = (const T *)a.hc + (size_t)m0 * a.d, rows_a = a.d;
        pb0 = (const T *)a.w + (size_t)(v0 + n0) * a.ws, rows_b = a.ws;
    } else if constexpr (KIND == DH) {
        pa0 = (const float *)a.grad + (size_t)m0 * a.piece, rows_a = a.piece;
        pb0 = (const T *)a.w + (size_t)v0 * a.ws + n0, step_b = a.ws;
    } else {
        pa0 = (const float *)a.grad + m0, step_a = a.piece;
        pb0 = (const T *)a.hc + n0, step_b = a.d;
    }
    const auto place = [&](bool mn, int x, int *k, int *m) {
        if (mn) *k = x / BM, *m = x % BM;
        else *k = (x & 7) + 8 * ((x >> 5) % (BK / 8)), *m = (x >> 3 & 3) + 4 * ((x >> 5) / (BK / 8));
    };
    const TA *pa[LOADS];
    const T *pb[LOADS];
    int ka[LOADS], kb[LOADS];  // the k of a thread's elements in front of k_hi, or none
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        int k, m;
        place(A_MN, tid + i * THREADS, &k, &m);
        pa[i] = pa0 + (size_t)m * rows_a + (size_t)(k_lo + k) * step_a;
        ka[i] = m0 + m < M ? k : 1 << 30;
        place(B_MN, tid + i * THREADS, &k, &m);
        pb[i] = pb0 + (size_t)m * rows_b + (size_t)(k_lo + k) * step_b;
        kb[i] = n0 + m < N ? k : 1 << 30;
    }
    float ra[LOADS], rb[LOADS];
    const auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            ra[i] = k0 + ka[i] < k_hi ? to_f(*pa[i]) : 0.f;
            rb[i] = k0 + kb[i] < k_hi ? to_f(*pb[i]) : 0.f;
            pa[i] += BK * step_a;
            pb[i] += BK * step_b;
        }
    };
    float c[E][E] = {};
    // (the error-free sum of two numbers, Knuth)
    const auto join = [&](bool first, bool last) {
#pragma unroll
        for (int i = 0; i < E; ++i)
#pragma unroll
            for (int j = 0; j < E; ++j) {
                float2 &r = runs[i * E + j][tid];
                const float2 w = first ? make_float2(0.f, 0.f) : r;
                const float t = w.x + c[i][j], y = t - w.x, cut = w.y + ((w.x - (t - y)) + (c[i][j] - y));
                c[i][j] = 0.f;
                if (last) c[i][j] = isfinite(cut) ? t + cut : t;
                else r = make_float2(t, cut);
            }
    };
    load(k_lo);
    int buf = 0;
    for (int k0 = k_lo; k0 < k_hi; k0 += BK, buf ^= 1) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int k, m;
            place(A_MN, tid + i * THREADS, &k, &m);
            s.a[buf][k][m] = ra[i];
            place(B_MN, tid + i * THREADS, &k, &m);
            s.b[buf][k][m] = rb[i];
        }
        __syncthreads();
        if (k0 + BK < k_hi) load(k0 + BK);
#pragma unroll
        for (int kk = 0; kk < BK / GROUPS; ++kk) {
            const int k = group * (BK / GROUPS) + kk;
            float xa[E], yb[E];
            if constexpr (E == 4) {
                const float4 x = *(const float4 *)&s.a[buf][k][ty * 4], y = *(const float4 *)&s.b[buf][k][tx * 4];
                xa[0] = x.x, xa[1] = x.y, xa[2] = x.z, xa[3] = x.w, yb[0] = y.x, yb[1] = y.y, yb[2] = y.z, yb[3] = y.w;
            } else {
                const float2 x = *(const float2 *)&s.a[buf][k][ty * 2], y = *(const float2 *)&s.b[buf][k][tx * 2];
                xa[0] = x.x, xa[1] = x.y, yb[0] = y.x, yb[1] = y.y;
            }
#pragma unroll
            for (int i = 0; i < E; ++i)
#pragma unroll
                for (int j = 0; j < E; ++j) c[i][j] = fmaf(xa[i], yb[j], c[i][j]);
        }
        if constexpr (KIND == DH || KIND == DW) {
            const int done = k0 + BK - k_lo;
            if (done % RUN == 0 && k0 + BK < k_hi) join(done == RUN, false);
        }
    }
    if constexpr (KIND == DH || KIND == DW) {
        if (k_hi - k_lo > RUN) join(false, true);
    }
    constexpr int MINE = E / GROUPS;  // rows of the tile that a thread is left with
    if constexpr (GROUPS > 1) {       // row 4 ty + group of each thread's four, from all groups
        float(*sum)[4][C::GROUP][4] = (float(*)[4][C::GROUP][4]) & s.a[0][0][0];
        static_assert(sizeof(float) * GROUPS * 4 * C::GROUP * 4 <= sizeof s.a + sizeof s.b, "sums");
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) *(float4 *)sum[group][i][at] = make_float4(c[i][0], c[i][1], c[i][2], c[i][3]);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) c[0][j] = 0.f;
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) {
            const float4 y = *(const float4 *)sum[q][group][at];
            c[0][0] += y.x, c[0][1] += y.y, c[0][2] += y.z, c[0][3] += y.w;
        }
    }
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        const int ml = ty * E + (GROUPS > 1 ? group : i), m = m0 + ml;
        if constexpr (KIND == LOSS) {
            // the threads of a row join their logits
            float mx = -INFINITY, l = 0.f;
            const int tgt = s.rows[ml].target;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int v = n0 + tx * E + j;
                if (v >= N) c[i][j] = -INFINITY;
                mx = fmaxf(mx, c[i][j]);
                if (v == tgt && m < M) a.at[m] = c[i][j];
            }
#pragma unroll
            for (int o = C::PER_ROW / 2; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float mu = mx == -INFINITY ? 0.f : mx;
#pragma unroll
            for (int j = 0; j < E; ++j) l += exp2f((c[i][j] - mu) * LOG2E);
#pragma unroll
            for (int o = C::PER_ROW / 2; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
            if (tx == 0 && m < M) a.part[(size_t)m * a.parts + n0 / BM] = make_float2(mx, l);
        } else {
            if (m >= M) continue;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int n = n0 + tx * E + j;
                if (n >= N) continue;
                if constexpr (KIND == GRAD) {
                    const VocabRow r = s.rows[ml];
                    const float p = exp2f((c[i][j] - r.lse) * LOG2E);
                    ((float *)a.grad)[(size_t)m * a.piece + n] = (v0 + n == r.target ? p - 1.f : p) * r.g;
                } else if constexpr (KIND == DH) {
                    float *to = a.acc + ((size_t)split * plane_rows + m) * a.d + n;
                    *to = v0 ? *to + c[i][j] : c[i][j];
                } else {
                    ((T *)a.dw)[(size_t)(v0 + m) * a.ws + n] = from_f<T>(c[i][j]);
                }
            }
        }
    }
}

// LOSS or GRAD.
template <typename T, int KIND, int BM>
__global__ void __launch_bounds__(THREADS) vocab_simt_kernel(const __grid_constant__ VocabArgs a, int v0) {
    __shared__ typename Simt<BM>::Smem s;
    pdl_wait();
    pdl_trigger();
    simt_tile<T, KIND, BM>(a, v0, blockIdx.x * BM, blockIdx.y * BM, 0, s);
}
// Both products of the gradient's piece: dh's tiles and splits, then dW's tiles.
template <typename T, int BM>
__global__ void __launch_bounds__(THREADS) vocab_simt_back_kernel(const __grid_constant__ VocabArgs a, int v0, int dh_blocks) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    typename Simt<BM>::BackSmem &s = *(typename Simt<BM>::BackSmem *)smem_raw;
    pdl_wait();
    pdl_trigger();
    const int i = blockIdx.x, n0 = blockIdx.y * BM;
    if (i < dh_blocks) {
        const int m_tiles = a.count->m_tiles, split = i / m_tiles;
        simt_tile<T, DH, BM>(a, v0, n0, (i - split * m_tiles) * BM, split, s, s.runs);
    } else {
        simt_tile<T, DW, BM>(a, v0, n0, (i - dh_blocks) * BM, 0, s, s.runs);
    }
}

template <typename T, int KIND, int BM>
cudaError_t run_simt(const VocabArgs &a, int v0, cudaStream_t st) {
    const int piece = a.V - v0 < a.piece ? a.V - v0 : a.piece;
    return launch_k(vocab_simt_kernel<T, KIND, BM>, dim3(ceil_div(piece, BM), ceil_div(a.n, BM)), dim3(THREADS), 0, st, a, v0);
}
template <typename T, int BM>
cudaError_t backward_simt(const VocabArgs &a, cudaStream_t st) {
    static bool known[MAX_DEVICES] = {};
    constexpr int bytes = (int)sizeof(typename Simt<BM>::BackSmem);
    const cudaError_t e0 = allow_smem(vocab_simt_back_kernel<T, BM>, bytes, known);
    if (e0 != cudaSuccess) return e0;
    for (int v0 = 0; v0 < a.V; v0 += a.piece) {
        cudaError_t e = run_simt<T, GRAD, BM>(a, v0, st);
        if (e != cudaSuccess) return e;
        // (as many as any count of tokens has: blocks of those that this one does not have leave)
        const int piece = a.V - v0 < a.piece ? a.V - v0 : a.piece, dh_blocks = (int)(a.acc_rows / BM);
        e = launch_k(vocab_simt_back_kernel<T, BM>, dim3(dh_blocks + (a.dw ? ceil_div(piece, BM) : 0), ceil_div(a.d, BM)), dim3(THREADS),
                     (size_t)bytes, st, a, v0, dh_blocks);
        if (e != cudaSuccess) return e;
        if (a.V - v0 <= a.piece) break;  // (v0 stays below 2^31)
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_vocab_keep(const VocabArgs &a, bool backward, cudaStream_t st) {
    // a warp a row, but no more than 1024 blocks, since each reads all targets
    const int per = a.n <= 1024 * WARPS ? WARPS : ceil_div(a.n, 1024);
    // (the rows to be cleared behind few tokens are shared by 32 blocks: 6 instead of 12 us)
    const int blocks = ceil_div(a.n, per);
    const dim3 grid(backward && a.tensor && blocks < 32 ? 32 : blocks);
    if (a.dtype == SP_F32) return launch_k(vocab_keep_kernel<float>, grid, dim3(THREADS), 0, st, a, per, (int)backward);
    return launch_k(vocab_keep_kernel<bf16>, grid, dim3(THREADS), 0, st, a, per, (int)backward);
}
cudaError_t launch_vocab_finish_loss(const VocabArgs &a, cudaStream_t st) {
    return launch_k(vocab_finish_loss_kernel, dim3(ceil_div(a.n, WARPS)), dim3(THREADS), 0, st, a);
}
cudaError_t launch_vocab_finish_dh(const VocabArgs &a, cudaStream_t st) {
    if (a.dtype == SP_F32) return launch_k(vocab_finish_dh_kernel<float>, dim3(a.n), dim3(THREADS), 0, st, a);
    return launch_k(vocab_finish_dh_kernel<bf16>, dim3(a.n), dim3(THREADS), 0, st, a);
}

// Tiles of 32 x 32 where 64 x 64 ones of the logits are fewer than the SMs (fp32, forward and backward, us: 250 tokens
// of 128 against 1000 rows 12 and 25, with 64 x 64 14 and 33; 100 of 512 against 2000 28 and 57, 33 and 56; 300 of
// 512 against 2000, 160 tiles, 55 and 103, 48 and 107; 500 of 512 against 4000 100 and 273, 85 and 226, which
// are 24 and 27 TFLOP/s, bound by reads of shared memory).  Pieces of the vocabulary
// whose gradients take at most 64 MB (or 64 rows), in whole tiles.
void plan_vocab_simt(VocabArgs *a, bool backward, int n_sm) {
    a->tm = (long long)ceil_div(a->n, 64) * ceil_div(a->V, 64) < n_sm ? 32 : 64;
    const int tm = a->tm;
    a->pad = a->n;
    a->pairs = 4 * n_sm;
    a->parts = ceil_div(a->V, tm);
    a->piece = ceil_div(a->V, tm) * tm;
    a->n_pieces = 1;
    if (backward) {
        long long most = (64ll << 20) / 4 / a->n / tm * tm;
        if (most > 65535ll * tm) most = 65535ll * tm;  // (tiles of M are the grid's second index)
        a->piece = most < tm ? tm : most < a->V ? (int)most : ceil_div(a->V, tm) * tm;
        a->n_pieces = ceil_div(a->V, a->piece);
    }
}

cudaError_t launch_vocab_loss_simt(const VocabArgs &a, cudaStream_t st) {
    if (a.dtype == SP_F32) return a.tm == 32 ? run_simt<float, LOSS, 32>(a, 0, st) : run_simt<float, LOSS, 64>(a, 0, st);
    return a.tm == 32 ? run_simt<bf16, LOSS, 32>(a, 0, st) : run_simt<bf16, LOSS, 64>(a, 0, st);
}
cudaError_t launch_vocab_backward_simt(const VocabArgs &a, cudaStream_t st) {
    if (a.dtype == SP_F32) return a.tm == 32 ? backward_simt<float, 32>(a, st) : backward_simt<float, 64>(a, st);
    return a.tm == 32 ? backward_simt<bf16, 32>(a, st) : backward_simt<bf16, 64>(a, st);
}

}  // namespace sp

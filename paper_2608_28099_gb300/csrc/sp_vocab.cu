// Cross entropy of tokens over a large vocabulary from the hidden states, and its gradients (the
// readout of a draft layer's hidden states by a language model's head, Sec. 3.1 and the head ablation
// of Sec. 5), without keeping the logits l = h W^T:
//   lse = log sum_v exp l_v,   loss = lse - l_t
//   g_v = dloss (exp(l_v - lse) - [v = t]),   dh = g W,   dW = g^T h
// Here: what stands around the products (counting off the tokens that have a target, joining the
// parts of a row's sum, writing gradients back to their tokens), and the products on CUDA cores in
// fp32 for fp32 rows and unaligned ones.  The tensor-core products are in sp_vocab_tc.cu.
#include "sp_train.cuh"

namespace sp {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int THREADS = 256, WARPS = THREADS / 32;

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
        if (threadIdx.x == 0) *a.count = all;
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
        if (p >= *a.count) return;
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
    if (p >= *a.count) return;
    T *to = (T *)a.dh + (size_t)a.rows[p].token * a.hs;
    const float *from = a.acc + (size_t)p * a.d;
    const DhPlan plan = dh_plan(a, *a.count);
    const size_t plane = (size_t)plan.rows * a.d;
    if (a.tensor) {  // (d a multiple of 8, rows aligned)
        for (int e = threadIdx.x * 4; e < a.d; e += THREADS * 4) {
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
            constexpr int AT_ONCE = 8;  // planes under way together
            for (int q0 = 0; q0 < plan.k.s; q0 += AT_ONCE) {
                float4 v[AT_ONCE];
#pragma unroll
                for (int q = 0; q < AT_ONCE; ++q)
                    v[q] = q0 + q < plan.k.s ? __ldcs((const float4 *)(from + (q0 + q) * plane + e)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int q = 0; q < AT_ONCE; ++q) s.x += v[q].x, s.y += v[q].y, s.z += v[q].z, s.w += v[q].w;
            }
            *(uint2 *)((bf16 *)to + e) = make_uint2(pack2_bf16(s.x, s.y), pack2_bf16(s.z, s.w));
        }
    } else {
        for (int e = threadIdx.x; e < a.d; e += THREADS) {
            float s = 0.f;
#pragma unroll 8
            for (int q = 0; q < plan.k.s; ++q) s += from[q * plane + e];
            to[e] = from_f<T>(s);
        }
    }
}

// ---------------------------------------------------------------------------
// Products on CUDA cores: C[m][n] = sum_k A(m, k) B(n, k) in 64 x 64 tiles, 32 of K at a time through
// two buffers in shared memory, the next ones' loads under way beside the products, 4 x 4 elements a
// thread, fp32 throughout; dh's tiles split along K where they are few.
enum { LOSS = 0, GRAD = 1, DH = 2, DW = 3 };
constexpr int BM = 64, BK = 32, LOADS = BM * BK / THREADS;

template <typename T, int KIND>
__global__ void __launch_bounds__(THREADS) vocab_simt_kernel(const __grid_constant__ VocabArgs a, int v0) {
    __shared__ float As[2][BK][BM + 4], Bs[2][BK][BM + 4];
    __shared__ VocabRow rows[BM];
    pdl_wait();
    pdl_trigger();
    const int count = *a.count;
    const int piece = min(a.piece, a.V - v0);
    // M, N, K of this product
    const int M = KIND == DW ? piece : count, N = KIND == LOSS || KIND == GRAD ? piece : a.d;
    const int K = KIND == DH ? piece : KIND == DW ? count : a.d;
    const int n0 = blockIdx.x * BM, m0 = blockIdx.y * BM;
    if (m0 >= M) return;
    int k_lo = 0, k_hi = K, plane_rows = 0;
    if (KIND == DH) {
        const DhPlan plan = dh_plan(a, count);
        if ((int)blockIdx.z >= plan.k.s) return;
        k_lo = min(K, (int)blockIdx.z * plan.k.per * BK);  // (the last piece may leave a split nothing: zeros)
        k_hi = min(K, k_lo + plan.k.per * BK);
        plane_rows = plan.rows;
    }
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    if (KIND != DW) {
        if (tid < BM) rows[tid] = m0 + tid < count ? a.rows[m0 + tid] : VocabRow{0.f, 0.f, -1, 0};
        __syncthreads();
    }
    const T *h = (const T *)a.hc, *w = (const T *)a.w;
    const float *grad = (const float *)a.grad;
    const auto A = [&](int m, int k) -> float {
        if (m0 + m >= M || k >= k_hi) return 0.f;
        if (KIND == LOSS || KIND == GRAD) return to_f(h[(size_t)(m0 + m) * a.d + k]);
        if (KIND == DH) return grad[(size_t)(m0 + m) * a.piece + k];
        return grad[(size_t)k * a.piece + m0 + m];
    };
    const auto B = [&](int n, int k) -> float {
        if (n0 + n >= N || k >= k_hi) return 0.f;
        if (KIND == LOSS || KIND == GRAD) return to_f(w[(size_t)(v0 + n0 + n) * a.ws + k]);
        if (KIND == DH) return to_f(w[(size_t)(v0 + k) * a.ws + n0 + n]);
        return to_f(h[(size_t)k * a.d + n0 + n]);
    };
    // neighbouring threads along whichever index is contiguous in memory
    const auto place = [&](bool mn, int x, int *k, int *m) { *k = mn ? x / BM : x % BK, *m = mn ? x % BM : x / BK; };
    float ra[LOADS], rb[LOADS];
    const auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int k, m;
            place(KIND == DW, tid + i * THREADS, &k, &m);
            ra[i] = A(m, k0 + k);
            place(KIND == DH || KIND == DW, tid + i * THREADS, &k, &m);
            rb[i] = B(m, k0 + k);
        }
    };
    float c[4][4] = {};
    load(k_lo);
    int buf = 0;
    for (int k0 = k_lo; k0 < k_hi; k0 += BK, buf ^= 1) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int k, m;
            place(KIND == DW, tid + i * THREADS, &k, &m);
            As[buf][k][m] = ra[i];
            place(KIND == DH || KIND == DW, tid + i * THREADS, &k, &m);
            Bs[buf][k][m] = rb[i];
        }
        __syncthreads();
        if (k0 + BK < k_hi) load(k0 + BK);
#pragma unroll
        for (int k = 0; k < BK; ++k) {
            const float4 x = *(const float4 *)&As[buf][k][ty * 4], y = *(const float4 *)&Bs[buf][k][tx * 4];
            const float xa[4] = {x.x, x.y, x.z, x.w}, yb[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) c[i][j] += xa[i] * yb[j];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int ml = ty * 4 + i, m = m0 + ml;
        if constexpr (KIND == LOSS) {
            // the 16 threads of a row join their 64 logits
            float mx = -INFINITY, l = 0.f;
            const int tgt = rows[ml].target;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int v = n0 + tx * 4 + j;
                if (v >= N) c[i][j] = -INFINITY;
                mx = fmaxf(mx, c[i][j]);
                if (v == tgt && m < M) a.at[m] = c[i][j];
            }
#pragma unroll
            for (int o = 8; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float mu = mx == -INFINITY ? 0.f : mx;
#pragma unroll
            for (int j = 0; j < 4; ++j) l += exp2f((c[i][j] - mu) * LOG2E);
#pragma unroll
            for (int o = 8; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
            if (tx == 0 && m < M) a.part[(size_t)m * a.parts + blockIdx.x] = make_float2(mx, l);
        } else {
            if (m >= M) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = n0 + tx * 4 + j;
                if (n >= N) continue;
                if constexpr (KIND == GRAD) {
                    const VocabRow r = rows[ml];
                    const float p = exp2f((c[i][j] - r.lse) * LOG2E);
                    ((float *)a.grad)[(size_t)m * a.piece + n] = (v0 + n == r.target ? p - 1.f : p) * r.g;
                } else if constexpr (KIND == DH) {
                    float *to = a.acc + ((size_t)blockIdx.z * plane_rows + m) * a.d + n;
                    *to = v0 ? *to + c[i][j] : c[i][j];
                } else {
                    ((T *)a.dw)[(size_t)(v0 + m) * a.ws + n] = from_f<T>(c[i][j]);
                }
            }
        }
    }
}

template <typename T, int KIND>
cudaError_t run_simt(const VocabArgs &a, int v0, cudaStream_t st) {
    const int piece = a.V - v0 < a.piece ? a.V - v0 : a.piece;
    const int M = KIND == DW ? piece : a.n, N = KIND == LOSS || KIND == GRAD ? piece : a.d;
    // (the splits for all counts: blocks of those that this one does not have leave)
    const int splits = KIND == DH ? 16 : 1;
    return launch_k(vocab_simt_kernel<T, KIND>, dim3(ceil_div(N, BM), ceil_div(M, BM), splits), dim3(THREADS), 0, st, a, v0);
}
template <typename T>
cudaError_t backward_simt(const VocabArgs &a, cudaStream_t st) {
    for (int v0 = 0; v0 < a.V; v0 += a.piece) {
        cudaError_t e = run_simt<T, GRAD>(a, v0, st);
        if (e == cudaSuccess) e = run_simt<T, DH>(a, v0, st);
        if (e == cudaSuccess && a.dw) e = run_simt<T, DW>(a, v0, st);
        if (e != cudaSuccess) return e;
        if (a.V - v0 <= a.piece) break;  // (v0 stays below 2^31)
    }
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_vocab_keep(const VocabArgs &a, bool backward, cudaStream_t st) {
    // a warp a row, but no more than 1024 blocks, since each reads all targets
    const int per = a.n <= 1024 * WARPS ? WARPS : ceil_div(a.n, 1024);
    return launch_k(a.dtype == SP_F32 ? vocab_keep_kernel<float> : vocab_keep_kernel<bf16>, dim3(ceil_div(a.n, per)), dim3(THREADS), 0,
                    st, a, per, (int)backward);
}
cudaError_t launch_vocab_finish_loss(const VocabArgs &a, cudaStream_t st) {
    return launch_k(vocab_finish_loss_kernel, dim3(ceil_div(a.n, WARPS)), dim3(THREADS), 0, st, a);
}
cudaError_t launch_vocab_finish_dh(const VocabArgs &a, cudaStream_t st) {
    return launch_k(a.dtype == SP_F32 ? vocab_finish_dh_kernel<float> : vocab_finish_dh_kernel<bf16>, dim3(a.n),
                    dim3(THREADS), 0, st, a);
}

// Pieces of the vocabulary whose gradients take at most 64 MB (or 64 rows), in whole tiles.
void plan_vocab_simt(VocabArgs *a, bool backward, int n_sm) {
    a->pad = a->n;
    a->pairs = 4 * n_sm;
    a->parts = ceil_div(a->V, BM);
    a->piece = ceil_div(a->V, BM) * BM;
    a->n_pieces = 1;
    if (backward) {
        long long most = (64ll << 20) / 4 / a->n / BM * BM;
        if (most > 65535ll * BM) most = 65535ll * BM;  // (tiles of M are the grid's second index)
        a->piece = most < BM ? BM : most < a->V ? (int)most : ceil_div(a->V, BM) * BM;
        a->n_pieces = ceil_div(a->V, a->piece);
    }
}

cudaError_t launch_vocab_loss_simt(const VocabArgs &a, cudaStream_t st) {
    return a.dtype == SP_F32 ? run_simt<float, LOSS>(a, 0, st) : run_simt<bf16, LOSS>(a, 0, st);
}
cudaError_t launch_vocab_backward_simt(const VocabArgs &a, cudaStream_t st) {
    return a.dtype == SP_F32 ? backward_simt<float>(a, st) : backward_simt<bf16>(a, st);
}

}  // namespace sp

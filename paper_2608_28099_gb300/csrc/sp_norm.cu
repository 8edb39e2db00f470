// Root-mean-square norm of rows, with a residual's addition in front of it and rows of
// fp32, bf16 or 8-bit codes behind it, and its backward pass (the norms of the decoder
// layer, Sec. 3.1):
//   s = x + r,  y = s rstd g,  rstd = (mean s^2 + eps)^-1/2
//   dx = rstd (g dy - xh m) + ds,  m = mean(g dy xh),  dg = sum over rows of dy xh,  xh = s rstd
// Both are bound by HBM: each row is read once into registers (8 elements a chunk, up to
// four chunks a thread) and one reduction over a row's threads stands between the loads and
// the stores.
#include "sp_train.cuh"

namespace sp {

namespace {

constexpr int MAX_CH = 4;        // 8-element chunks of a row a thread holds
constexpr int LOOP_THREADS = 256;

// rstd as a power of two times a float: rows whose squares leave fp32 still have a norm.
struct Rstd {
    float f1, f2;
    __device__ __forceinline__ float of(float v) const { return v * f1 * f2; }
};
__device__ __forceinline__ Rstd rstd_of(double mean_sq) {
    const double r = rsqrt(mean_sq);
    if (!(r > 0.0 && r < 1e60)) return Rstd{1.f, (float)r};
    int e;
    frexp(r, &e);
    e = min(max(e, -126), 127);
    return Rstd{(float)ldexp(1.0, e), (float)ldexp(r, -e)};
}
// Whether the fp32 sum of squares cannot be relied on: squares beyond fp32, or lost
// below it with no eps that would hide them.
__device__ __forceinline__ bool out_of_range(float sq, float eps) {
    return sq > 1.3e36f || (sq < 8.7e-19f && eps < 9.1e-13f);  // (2^120, 2^-60, 2^-40)
}

// Sums (or maxima) of two values over the TPR threads of a row; every thread gets them.
template <int TPR, bool MAX = false, typename T>
__device__ __forceinline__ void reduce2(T &a, T &b, T (*buf)[2]) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const T x = __shfl_xor_sync(0xffffffffu, a, o), y = __shfl_xor_sync(0xffffffffu, b, o);
        a = MAX ? max(a, x) : a + x;
        b = MAX ? max(b, y) : b + y;
    }
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        const int warp = threadIdx.x >> 5, first = warp / W * W;
        __syncthreads();  // (an earlier use is read)
        if ((threadIdx.x & 31) == 0) buf[warp][0] = a, buf[warp][1] = b;
        __syncthreads();
        a = buf[first][0], b = buf[first][1];
#pragma unroll
        for (int w = 1; w < W; ++w) {
            a = MAX ? max(a, buf[first + w][0]) : a + buf[first + w][0];
            b = MAX ? max(b, buf[first + w][1]) : b + buf[first + w][1];
        }
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
        *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
        *(float4 *)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *(uint4 *)p = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
    }
}
__device__ __forceinline__ void gain8(const float *g, int e, float (&v)[8]) {
    if (g) {
        load8(g + e, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.f;
    }
}
// The 8-bit code of a value times the row's factor; what is not finite becomes NaN.
__device__ __forceinline__ float code_in(float v, float f) { return isfinite(v) ? v * f : NAN; }

// TPR threads a row, CH chunks a thread.
template <typename T, int TPR, int CH, bool E8>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) norm_kernel(const __grid_constant__ NormArgs a) {
    constexpr int BLOCK = TPR < 128 ? 128 : TPR;
    __shared__ float buf[BLOCK / 32][2];
    __shared__ double dbuf[BLOCK / 32][2];
    pdl_wait();
    pdl_trigger();
    const int t = threadIdx.x % TPR;
    const long long row = (long long)blockIdx.x * (BLOCK / TPR) + threadIdx.x / TPR;
    const bool live = row < a.n;
    float v[CH][8];
    float sq = 0.f, none = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * TPR + t) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] = 0.f;
        if (live && e < a.d) load8((const T *)a.x + row * a.xs + e, v[c]);
    }
    if (a.r) {
        float r[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * TPR + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) r[c][i] = 0.f;
            if (live && e < a.d) load8((const T *)a.r + row * a.rs + e, r[c]);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] += r[c][i];
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) sq += v[c][i] * v[c][i];
    reduce2<TPR>(sq, none, buf);
    Rstd rs{1.f, rsqrtf(sq / (float)a.d + a.eps)};
    // (a verdict of the block: reduce2 meets at its barriers)
    if (__syncthreads_or(out_of_range(sq, a.eps))) {
        double q = 0.0, z = 0.0;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) q += (double)v[c][i] * v[c][i];
        reduce2<TPR>(q, z, dbuf);
        if (out_of_range(sq, a.eps)) rs = rstd_of(q / a.d + a.eps);
    }
    float amax = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * TPR + t) * 8;
        if (!live || e >= a.d) continue;
        if (a.sum) store8((T *)a.sum + row * a.ss + e, v[c]);
        float g[8];
        gain8(a.gain, e, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[c][i] = rs.of(v[c][i]) * g[i];
            if (E8 && isfinite(v[c][i])) amax = fmaxf(amax, fabsf(v[c][i]));
        }
        if constexpr (!E8) store8((T *)a.y + row * a.ys + e, v[c]);
    }
    if constexpr (E8) {
        reduce2<TPR, true>(amax, none, buf);
        amax = fmaxf(amax, kMinAmax);
        const float f = kMaxCode / amax;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * TPR + t) * 8;
            if (!live || e >= a.d) continue;
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = float_to_codes2(code_in(v[c][2 * i], f), code_in(v[c][2 * i + 1], f));
            *(uint2 *)((uint8_t *)a.y + row * a.ys + e) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
        }
        if (live && t == 0) a.y_scale[row] = amax * (1.f / kMaxCode);
    }
}

// Rows of any length and alignment: an element a thread, the row read again for each use.
template <typename T>
__global__ void __launch_bounds__(LOOP_THREADS) norm_loop_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float buf[LOOP_THREADS / 32][2];
    __shared__ double dbuf[LOOP_THREADS / 32][2];
    pdl_wait();
    pdl_trigger();
    const long long row = blockIdx.x;
    const T *x = (const T *)a.x + row * a.xs, *r = a.r ? (const T *)a.r + row * a.rs : nullptr;
    const auto value = [&](int e) { return to_f(x[e]) + (r ? to_f(r[e]) : 0.f); };
    const auto normed = [&](float v, const Rstd &rs, int e) { return rs.of(v) * (a.gain ? a.gain[e] : 1.f); };
    float sq = 0.f, none = 0.f;
    for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) {
        const float v = value(e);
        sq += v * v;
    }
    reduce2<LOOP_THREADS>(sq, none, buf);
    Rstd rs{1.f, rsqrtf(sq / (float)a.d + a.eps)};
    if (out_of_range(sq, a.eps)) {  // (the same for all threads)
        double q = 0.0, z = 0.0;
        for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) {
            const double v = value(e);
            q += v * v;
        }
        reduce2<LOOP_THREADS>(q, z, dbuf);
        rs = rstd_of(q / a.d + a.eps);
    }
    float amax = 0.f;
    const bool e8 = a.out_dtype == SP_E4M3;
    if (e8) {
        for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) {
            const float y = normed(value(e), rs, e);
            if (isfinite(y)) amax = fmaxf(amax, fabsf(y));
        }
        reduce2<LOOP_THREADS, true>(amax, none, buf);
        amax = fmaxf(amax, kMinAmax);
        if (threadIdx.x == 0) a.y_scale[row] = amax * (1.f / kMaxCode);
    }
    const float f = e8 ? kMaxCode / amax : 1.f;
    for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) {
        const float v = value(e), y = normed(v, rs, e);
        if (a.sum) ((T *)a.sum)[row * a.ss + e] = from_f<T>(v);
        if (e8) ((uint8_t *)a.y)[row * a.ys + e] = (uint8_t)float_to_codes2(code_in(y, f), 0.f);
        else ((T *)a.y)[row * a.ys + e] = from_f<T>(y);
    }
}

// Backward: a block walks rows gridDim apart; a thread keeps its columns' part of the gain's gradient.
template <typename T, int TPR, int CH>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) norm_back_kernel(const __grid_constant__ NormBackArgs a) {
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, RPB = BLOCK / TPR;
    __shared__ float buf[BLOCK / 32][2];
    __shared__ double dbuf[BLOCK / 32][2];
    pdl_wait();
    pdl_trigger();
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    float dg[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[c][i] = 0.f;
    // (the same number of steps for all threads: they meet at barriers)
    for (long long first = (long long)blockIdx.x * RPB; first < a.n; first += (long long)gridDim.x * RPB) {
        const long long row = first + sub;
        const bool live = row < a.n;
        float s[CH][8], y[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * TPR + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) s[c][i] = y[c][i] = 0.f;
            if (live && e < a.d) {
                load8((const T *)a.s + row * a.ss + e, s[c]);
                load8((const T *)a.dy + row * a.ys + e, y[c]);
            }
        }
        float sq = 0.f, dot = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * TPR + t) * 8;
            float g[8];
            if (e < a.d) gain8(a.gain, e, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (e >= a.d) g[i] = 0.f;
                sq += s[c][i] * s[c][i];
                dot += y[c][i] * g[i] * s[c][i];
            }
        }
        reduce2<TPR>(sq, dot, buf);
        Rstd rs{1.f, rsqrtf(sq / (float)a.d + a.eps)};
        float m = rs.f2 * dot / (float)a.d;
        if (__syncthreads_or(out_of_range(sq, a.eps) || !isfinite(m))) {
            double q = 0.0, z = 0.0;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int e = (c * TPR + t) * 8;
                float g[8];
                if (e < a.d) gain8(a.gain, e, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q += (double)s[c][i] * s[c][i];
                    if (e < a.d) z += (double)y[c][i] * g[i] * s[c][i];
                }
            }
            reduce2<TPR>(q, z, dbuf);
            if (out_of_range(sq, a.eps) || !isfinite(m)) {
                rs = rstd_of(q / a.d + a.eps);
                m = (float)(z / a.d * rs.f1 * rs.f2);
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * TPR + t) * 8;
            if (!live || e >= a.d) continue;
            float g[8], ds[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (a.ds) load8((const T *)a.ds + row * a.rs + e, ds);
            gain8(a.gain, e, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float xh = rs.of(s[c][i]);
                dg[c][i] += y[c][i] * xh;
                ds[i] += rs.of(y[c][i] * g[i] - xh * m);
            }
            store8((T *)a.dx + row * a.xs + e, ds);
        }
    }
    if (a.dgain) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * TPR + t) * 8;
            if (e < a.d) store8(a.part + ((size_t)blockIdx.x * RPB + sub) * a.d + e, dg[c]);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(LOOP_THREADS) norm_back_loop_kernel(const __grid_constant__ NormBackArgs a) {
    __shared__ float buf[LOOP_THREADS / 32][2];
    __shared__ double dbuf[LOOP_THREADS / 32][2];
    pdl_wait();
    pdl_trigger();
    float *part = a.part + (size_t)blockIdx.x * a.d;
    if (a.dgain)
        for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) part[e] = 0.f;
    for (long long row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T *s = (const T *)a.s + row * a.ss, *dy = (const T *)a.dy + row * a.ys;
        float sq = 0.f, dot = 0.f;
        for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) {
            const float v = to_f(s[e]);
            sq += v * v;
            dot += to_f(dy[e]) * (a.gain ? a.gain[e] : 1.f) * v;
        }
        reduce2<LOOP_THREADS>(sq, dot, buf);
        Rstd rs{1.f, rsqrtf(sq / (float)a.d + a.eps)};
        float m = rs.f2 * dot / (float)a.d;
        if (out_of_range(sq, a.eps) || !isfinite(m)) {  // (the same for all threads)
            double q = 0.0, z = 0.0;
            for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) {
                const double v = to_f(s[e]);
                q += v * v;
                z += (double)to_f(dy[e]) * (a.gain ? a.gain[e] : 1.f) * v;
            }
            reduce2<LOOP_THREADS>(q, z, dbuf);
            rs = rstd_of(q / a.d + a.eps);
            m = (float)(z / a.d * rs.f1 * rs.f2);
        }
        for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) {
            const float xh = rs.of(to_f(s[e])), y = to_f(dy[e]);
            const float ds = a.ds ? to_f(((const T *)a.ds)[row * a.rs + e]) : 0.f;
            if (a.dgain) part[e] += y * xh;
            ((T *)a.dx)[row * a.xs + e] = from_f<T>(ds + rs.of(y * (a.gain ? a.gain[e] : 1.f) - xh * m));
        }
    }
}

// dg: the partial rows added in their order, a column a thread of the first warp's
// lanes, the rows split over eight warps whose sums are added in order.
constexpr int SUM_WARPS = 8;
__global__ void __launch_bounds__(32 * SUM_WARPS) norm_gain_kernel(const float *part, int parts, int d, float *dgain) {
    __shared__ float sums[SUM_WARPS][32];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    const int per = ceil_div(parts, SUM_WARPS), lo = warp * per, hi = min(parts, lo + per);
    float s = 0.f;
    if (e < d) {
#pragma unroll 8
        for (int p = lo; p < hi; ++p) s += part[(size_t)p * d + e];
    }
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && e < d) {
#pragma unroll
        for (int w = 1; w < SUM_WARPS; ++w) s += sums[w][lane];
        dgain[e] = s;
    }
}

// Threads a row and chunks a thread: the fewest threads (a multiple of a warp, a power of two) that
// hold a row in up to four chunks; 0: too long.
struct Shape {
    int tpr, ch;
};
Shape shape_of(int d) {
    const int chunks = ceil_div(d, 8);
    int tpr = 32;
    while (tpr < 1024 && tpr * 2 < chunks) tpr *= 2;  // two chunks a thread until 1024 threads
    const int ch = ceil_div(chunks, tpr);
    return Shape{ch <= MAX_CH ? tpr : 0, ch <= 1 ? 1 : ch <= 2 ? 2 : 4};
}
bool whole16(const void *p, long long stride, int es) { return !(((uintptr_t)p | (uintptr_t)(stride * es)) & 15); }

template <typename T, int TPR, int CH>
cudaError_t run_norm(const NormArgs &a, cudaStream_t st) {
    constexpr int BLOCK = TPR < 128 ? 128 : TPR;
    const dim3 grid((unsigned)ceil_div_ll(a.n, BLOCK / TPR));
    if (a.out_dtype == SP_E4M3) return launch_k(norm_kernel<T, TPR, CH, true>, grid, dim3(BLOCK), 0, st, a);
    return launch_k(norm_kernel<T, TPR, CH, false>, grid, dim3(BLOCK), 0, st, a);
}
template <typename T, int TPR, int CH>
cudaError_t run_back(const NormBackArgs &a, int parts, cudaStream_t st) {
    constexpr int BLOCK = TPR < 128 ? 128 : TPR;
    return launch_k(norm_back_kernel<T, TPR, CH>, dim3(parts / (BLOCK / TPR)), dim3(BLOCK), 0, st, a);
}
// f(TPR, CH) of a shape
#define SP_NORM_SHAPES(CALL)                                                                       \
    switch (s.tpr) {                                                                               \
    case 32: return s.ch == 1 ? CALL(32, 1) : CALL(32, 2);                                         \
    case 64: return CALL(64, 2);                                                                   \
    case 128: return CALL(128, 2);                                                                 \
    case 256: return CALL(256, 2);                                                                 \
    case 512: return CALL(512, 2);                                                                 \
    default: return s.ch <= 2 ? CALL(1024, 2) : CALL(1024, 4);                                     \
    }
template <typename T>
cudaError_t norm_shapes(const NormArgs &a, Shape s, cudaStream_t st) {
#define SP_CALL(TPR, CH) run_norm<T, TPR, CH>(a, st)
    SP_NORM_SHAPES(SP_CALL)
#undef SP_CALL
}
template <typename T>
cudaError_t back_shapes(const NormBackArgs &a, Shape s, int parts, cudaStream_t st) {
#define SP_CALL(TPR, CH) run_back<T, TPR, CH>(a, parts, st)
    SP_NORM_SHAPES(SP_CALL)
#undef SP_CALL
}
#undef SP_NORM_SHAPES

}  // namespace

cudaError_t launch_norm(const NormArgs &a, cudaStream_t st) {
    const int es = a.dtype == SP_F32 ? 4 : 2;
    const bool e8 = a.out_dtype == SP_E4M3;
    const bool y_whole = e8 ? !(((uintptr_t)a.y | (uintptr_t)a.ys) & 7) : whole16(a.y, a.ys, es);
    const bool vec = a.d % 8 == 0 && whole16(a.x, a.xs, es) && (!a.r || whole16(a.r, a.rs, es)) &&
                     (!a.sum || whole16(a.sum, a.ss, es)) && y_whole && whole16(a.gain, 0, 4);
    const Shape s = shape_of(a.d);
    if (!vec || !s.tpr) {
        if (a.dtype == SP_F32) return launch_k(norm_loop_kernel<float>, dim3(a.n), dim3(LOOP_THREADS), 0, st, a);
        return launch_k(norm_loop_kernel<bf16>, dim3(a.n), dim3(LOOP_THREADS), 0, st, a);
    }
    return a.dtype == SP_F32 ? norm_shapes<float>(a, s, st) : norm_shapes<bf16>(a, s, st);
}

// A multiple of the rows that a block takes at once, for both kinds of kernel.
int norm_back_parts(int n, int d, int n_sm) {
    const Shape s = shape_of(d);
    const int tpr = s.tpr ? s.tpr : LOOP_THREADS, rpb = tpr < 128 ? 128 / tpr : 1;
    const int per_sm = tpr <= 128 ? 8 : tpr >= 1024 ? 1 : 1024 / tpr;
    const long long blocks = ceil_div_ll(n, rpb);
    return (int)(blocks < (long long)n_sm * per_sm ? blocks : (long long)n_sm * per_sm) * rpb;
}

cudaError_t launch_norm_backward(const NormBackArgs &a, int n_sm, cudaStream_t st) {
    const int es = a.dtype == SP_F32 ? 4 : 2;
    const bool vec = a.d % 8 == 0 && whole16(a.dx, a.xs, es) && (!a.ds || whole16(a.ds, a.rs, es)) &&
                     whole16(a.s, a.ss, es) && whole16(a.dy, a.ys, es) && whole16(a.gain, 0, 4);
    const Shape s = shape_of(a.d);
    const int parts = norm_back_parts(a.n, a.d, n_sm);
    cudaError_t e;
    if (!vec || !s.tpr) {
        const auto k = a.dtype == SP_F32 ? norm_back_loop_kernel<float> : norm_back_loop_kernel<bf16>;
        e = launch_k(k, dim3(parts), dim3(LOOP_THREADS), 0, st, a);
    } else {
        e = a.dtype == SP_F32 ? back_shapes<float>(a, s, parts, st) : back_shapes<bf16>(a, s, parts, st);
    }
    if (e != cudaSuccess || !a.dgain) return e;
    return launch_k(norm_gain_kernel, dim3(ceil_div(a.d, 32)), dim3(32 * SUM_WARPS), 0, st, (const float *)a.part, parts, a.d,
                    a.dgain);
}

}  // namespace sp

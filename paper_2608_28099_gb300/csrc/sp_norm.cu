// Root-mean-square norm of rows, with a residual's addition in front of it and rows of
// fp32, bf16 or 8-bit codes behind it, and its backward pass (the norms of the decoder
// layer, Sec. 3.1):
//   s = x + r,  y = s rstd g,  rstd = (mean s^2 + eps)^-1/2
//   dx = rstd (g dy - xh m) + ds,  m = mean(g dy xh),  dg = sum over rows of dy xh,  xh = s rstd
// Both are bound by HBM: each row is read once into registers (8 elements a chunk, up to four chunks a
// thread) and one reduction over a row's threads stands between the loads and the stores, so blocks walk
// rows and have the next one's loads under way meanwhile (without: 143 instead of 99 us, 94 instead
// of 49).  16384 rows of 5120, bf16 with a residual into 8 bits: 99 us, 5.9 TB/s; backward of 8191 rows of
// 4096 with the gain's gradient 49 us, 5.5 TB/s, 5 of them its second kernel; of 1500 fp32 rows of 2560
// without it 12.9 us, 4.8 TB/s: its registers let three blocks of 160 threads onto an SM where the grid has four, so that
// 456 of the 608 blocks run first and the others behind them.  16 rows of 4096: 4.3 us, one launch.
#include "sp_train.cuh"

namespace sp {

namespace {

constexpr int LOOP_THREADS = 256, MAX_THREADS = 512;
// Rows of any length: a thread adds RUN terms after one another and its runs with what each addition cuts off, so
// that a sum's error does not grow with the row (2^24 equal elements, 65536 a thread, added up in one fp32
// number: norms off by 3e-4).
constexpr int RUN = 16;

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

// Sums (or maxima) of two values over the threads of a row (a warp, or WARP = false: the block);
// every thread gets them.  Uses of buf one after another alternate between its halves: a barrier a use.
template <bool WARP, bool MAX = false, typename T>
__device__ __forceinline__ void reduce2(T &a, T &b, T (*buf)[32][2], int &half) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const T x = __shfl_xor_sync(0xffffffffu, a, o), y = __shfl_xor_sync(0xffffffffu, b, o);
        a = MAX ? max(a, x) : a + x;
        b = MAX ? max(b, y) : b + y;
    }
    if constexpr (!WARP) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
        if (lane == 0) buf[half][warp][0] = a, buf[half][warp][1] = b;
        __syncthreads();
        a = lane < warps ? buf[half][lane][0] : T(0), b = lane < warps ? buf[half][lane][1] : T(0);  // (maxima are >= 0)
        half ^= 1;
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const T x = __shfl_xor_sync(0xffffffffu, a, o), y = __shfl_xor_sync(0xffffffffu, b, o);
            a = MAX ? max(a, x) : a + x;
            b = MAX ? max(b, y) : b + y;
        }
    }
}

// A sum that keeps what its additions cut off (the error-free sum of two numbers, Knuth).
struct Sum {
    float s = 0.f, cut = 0.f;
    __device__ __forceinline__ void add(float x) {
        const float t = s + x, y = t - s;
        cut += (s - (t - y)) + (x - y);
        s = t;
    }
    __device__ __forceinline__ float get() const { return isfinite(cut) ? s + cut : s; }  // (beyond fp32: as it is)
};
// A thread's part of a row's sums of two terms of each element.
template <typename F>
__device__ __forceinline__ float2 thread_sums(int d, const F &term) {
    int e = threadIdx.x;
    Sum a, b;
    for (; e < d - (RUN - 1) * LOOP_THREADS; e += RUN * LOOP_THREADS) {
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int i = 0; i < RUN; ++i) term(e + i * LOOP_THREADS, x, y);
        a.add(x);
        b.add(y);
    }
    float x = 0.f, y = 0.f;
    for (; e < d; e += LOOP_THREADS) term(e, x, y);
    if (d <= (RUN - 1) * LOOP_THREADS) return make_float2(x, y);
    a.add(x);
    b.add(y);
    return make_float2(a.get(), b.get());
}

// Eight elements as they lie in memory.
template <typename T>
struct Raw {
    uint4 u[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) u[i] = *(const uint4 *)(p + i * (16 / (int)sizeof(T)));
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) u[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        if constexpr (sizeof(T) == 4) {
            v[0] = __uint_as_float(u[0].x), v[1] = __uint_as_float(u[0].y), v[2] = __uint_as_float(u[0].z), v[3] = __uint_as_float(u[0].w);
            v[4] = __uint_as_float(u[1].x), v[5] = __uint_as_float(u[1].y), v[6] = __uint_as_float(u[1].z), v[7] = __uint_as_float(u[1].w);
        } else {
            const uint32_t w[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
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

// A row a block (WARP: a warp), CH chunks a thread; rows gridDim apart, the next one's loads under
// way while this one is reduced and written.
template <typename T, bool WARP, int CH, bool E8>
__global__ void __launch_bounds__(WARP ? 128 : MAX_THREADS) norm_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float buf[2][32][2];
    __shared__ double dbuf[2][32][2];
    int half = 0, dhalf = 0;
    pdl_wait();
    pdl_trigger();
    const int tpr = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x & 31 : threadIdx.x;
    const int rows_b = WARP ? blockDim.x >> 5 : 1;
    const long long step = (long long)gridDim.x * rows_b;
    long long row = (long long)blockIdx.x * rows_b + (WARP ? threadIdx.x >> 5 : 0);
    Raw<T> x[CH], r[CH];
    const auto load = [&](long long at) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * tpr + t) * 8;
            x[c].zero();
            r[c].zero();
            if (e < a.d) {
                x[c].load((const T *)a.x + at * a.xs + e);
                if (a.r) r[c].load((const T *)a.r + at * a.rs + e);
            }
        }
    };
    if (row < a.n) load(row);
    for (; row < a.n; row += step) {
        float v[CH][8];
        float sq = 0.f, none = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float z[8];
            x[c].get(v[c]);
            r[c].get(z);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[c][i] += z[i];
                sq += v[c][i] * v[c][i];
            }
        }
        if (row + step < a.n) load(row + step);
        reduce2<WARP>(sq, none, buf, half);
        Rstd rs{1.f, rsqrtf(sq / (float)a.d + a.eps)};
        if (out_of_range(sq, a.eps)) {  // (the same for the row's threads)
            double q = 0.0, z = 0.0;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) q += (double)v[c][i] * v[c][i];
            reduce2<WARP>(q, z, dbuf, dhalf);
            rs = rstd_of(q / a.d + a.eps);
        }
        float amax = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * tpr + t) * 8;
            if (e >= a.d) continue;
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
            reduce2<WARP, true>(amax, none, buf, half);
            amax = fmaxf(amax, kMinAmax);
            const float f = kMaxCode / amax;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int e = (c * tpr + t) * 8;
                if (e >= a.d) continue;
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = float_to_codes2(code_in(v[c][2 * i], f), code_in(v[c][2 * i + 1], f));
                *(uint2 *)((uint8_t *)a.y + row * a.ys + e) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
            }
            if (t == 0) a.y_scale[row] = amax * (1.f / kMaxCode);
        }
    }
}

// Rows of any length and alignment: an element a thread, the row read again for each use.
template <typename T>
__global__ void __launch_bounds__(LOOP_THREADS) norm_loop_kernel(const __grid_constant__ NormArgs a) {
    __shared__ float buf[2][32][2];
    __shared__ double dbuf[2][32][2];
    int half = 0, dhalf = 0;
    pdl_wait();
    pdl_trigger();
    const long long row = blockIdx.x;
    const T *x = (const T *)a.x + row * a.xs, *r = a.r ? (const T *)a.r + row * a.rs : nullptr;
    const auto value = [&](int e) { return to_f(x[e]) + (r ? to_f(r[e]) : 0.f); };
    const auto normed = [&](float v, const Rstd &rs, int e) { return rs.of(v) * (a.gain ? a.gain[e] : 1.f); };
    float none = 0.f, sq = thread_sums(a.d, [&](int e, float &x, float &) {
        const float v = value(e);
        x += v * v;
    }).x;
    reduce2<false>(sq, none, buf, half);
    Rstd rs{1.f, rsqrtf(sq / (float)a.d + a.eps)};
    if (out_of_range(sq, a.eps)) {  // (the same for all threads)
        double q = 0.0, z = 0.0;
        for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) {
            const double v = value(e);
            q += v * v;
        }
        reduce2<false>(q, z, dbuf, dhalf);
        rs = rstd_of(q / a.d + a.eps);
    }
    float amax = 0.f;
    const bool e8 = a.out_dtype == SP_E4M3;
    if (e8) {
        for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) {
            const float y = normed(value(e), rs, e);
            if (isfinite(y)) amax = fmaxf(amax, fabsf(y));
        }
        reduce2<false, true>(amax, none, buf, half);
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

// Backward, likewise; a thread keeps its columns' part of the gain's gradient, and the gain.
template <typename T, bool WARP, int CH>
__global__ void __launch_bounds__(WARP ? 128 : MAX_THREADS) norm_back_kernel(const __grid_constant__ NormBackArgs a) {
    __shared__ float buf[2][32][2];
    __shared__ double dbuf[2][32][2];
    int half = 0, dhalf = 0;
    pdl_wait();
    pdl_trigger();
    const int tpr = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x & 31 : threadIdx.x;
    const int rows_b = WARP ? blockDim.x >> 5 : 1;
    const long long step = (long long)gridDim.x * rows_b;
    const long long first = (long long)blockIdx.x * rows_b + (WARP ? threadIdx.x >> 5 : 0);
    float dg[CH][8], g[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * tpr + t) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[c][i] = g[c][i] = 0.f;
        if (e < a.d) gain8(a.gain, e, g[c]);
    }
    Raw<T> rs_[CH], ry[CH], rd[CH];
    const auto load = [&](long long at) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * tpr + t) * 8;
            rs_[c].zero();
            ry[c].zero();
            if (e < a.d) {
                rs_[c].load((const T *)a.s + at * a.ss + e);
                ry[c].load((const T *)a.dy + at * a.ys + e);
            }
        }
    };
    if (first < a.n) load(first);
    for (long long row = first; row < a.n; row += step) {
        float s[CH][8], y[CH][8];
        float sq = 0.f, dot = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * tpr + t) * 8;
            rd[c].zero();
            if (a.ds && e < a.d) rd[c].load((const T *)a.ds + row * a.rs + e);
            rs_[c].get(s[c]);
            ry[c].get(y[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sq += s[c][i] * s[c][i];
                dot += y[c][i] * g[c][i] * s[c][i];
            }
        }
        if (row + step < a.n) load(row + step);
        reduce2<WARP>(sq, dot, buf, half);
        Rstd rs{1.f, rsqrtf(sq / (float)a.d + a.eps)};
        float m = rs.f2 * dot / (float)a.d;
        if (out_of_range(sq, a.eps) || !isfinite(m)) {  // (the same for the row's threads)
            double q = 0.0, z = 0.0;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q += (double)s[c][i] * s[c][i];
                    z += (double)y[c][i] * g[c][i] * s[c][i];
                }
            reduce2<WARP>(q, z, dbuf, dhalf);
            rs = rstd_of(q / a.d + a.eps);
            m = (float)(z / a.d * rs.f1 * rs.f2);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * tpr + t) * 8;
            float ds[8];
            rd[c].get(ds);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float xh = rs.of(s[c][i]);
                dg[c][i] += y[c][i] * xh;
                ds[i] += rs.of(y[c][i] * g[c][i] - xh * m);
            }
            if (e < a.d) store8((T *)a.dx + row * a.xs + e, ds);
        }
    }
    if (a.dgain) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * tpr + t) * 8;
            if (e < a.d) store8(a.part + first * a.d + e, dg[c]);
        }
    }
}

template <typename T>
struct LoopRow {
    const T *s, *dy, *ds;
    T *dx;
    __device__ __forceinline__ LoopRow(const NormBackArgs &a, long long row)
        : s((const T *)a.s + row * a.ss), dy((const T *)a.dy + row * a.ys), ds(a.ds ? (const T *)a.ds + row * a.rs : nullptr),
          dx((T *)a.dx + row * a.xs) {}
    // dx of an element, in front of whose store `keep` takes its part of the gain's gradient
    template <typename F>
    __device__ __forceinline__ void element(int e, float gain, const Rstd &rs, float m, const F &keep) const {
        const float xh = rs.of(to_f(s[e])), y = to_f(dy[e]), z = ds ? to_f(ds[e]) : 0.f;
        keep(y * xh);
        dx[e] = from_f<T>(z + rs.of(y * gain - xh * m));
    }
};
template <typename T>
__global__ void __launch_bounds__(LOOP_THREADS) norm_back_loop_kernel(const __grid_constant__ NormBackArgs a) {
    __shared__ float buf[2][32][2];
    __shared__ double dbuf[2][32][2];
    int half = 0, dhalf = 0;
    pdl_wait();
    pdl_trigger();
    const auto gain = [&](int e) { return a.gain ? a.gain[e] : 1.f; };
    float *part = a.part + (size_t)blockIdx.x * a.d;
    if (a.dgain)
        for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) part[e] = 0.f;
    for (long long row = blockIdx.x; row < a.n; row += gridDim.x) {
        const LoopRow<T> r(a, row);
        const float2 mine = thread_sums(a.d, [&](int e, float &x, float &y) {
            const float v = to_f(r.s[e]);
            x += v * v;
            y += to_f(r.dy[e]) * gain(e) * v;
        });
        float sq = mine.x, dot = mine.y;
        reduce2<false>(sq, dot, buf, half);
        Rstd rs{1.f, rsqrtf(sq / (float)a.d + a.eps)};
        float m = rs.f2 * dot / (float)a.d;
        if (out_of_range(sq, a.eps) || !isfinite(m)) {  // (the same for all threads)
            double q = 0.0, z = 0.0;
            for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS) {
                const double v = to_f(r.s[e]);
                q += v * v;
                z += (double)to_f(r.dy[e]) * gain(e) * v;
            }
            reduce2<false>(q, z, dbuf, dhalf);
            rs = rstd_of(q / a.d + a.eps);
            m = (float)(z / a.d * rs.f1 * rs.f2);
        }
        for (int e = threadIdx.x; e < a.d; e += LOOP_THREADS)
            r.element(e, gain(e), rs, m, [&](float dg) {
                if (a.dgain) part[e] += dg;
            });
    }
}

// dg: the partial rows added in their order, a column a thread of the first warp's
// lanes, the rows split over 32 warps whose sums are added in pairs.  more: dg holds the sum of rows in front.
constexpr int SUM_WARPS = 32, FEW_PARTS = 20;
__global__ void __launch_bounds__(32 * SUM_WARPS) norm_gain_kernel(const float *part, int parts, int d, float *dgain, int more) {
    __shared__ float sums[SUM_WARPS][32];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    const int per = ceil_div(parts, SUM_WARPS), lo = warp * per, hi = min(parts, lo + per);
    float s = 0.f;
    if (e < d && per <= FEW_PARTS) {
#pragma unroll 8
        for (int p = lo; p < hi; ++p) s += part[(size_t)p * d + e];
    } else if (e < d) {
        Sum many;
#pragma unroll 8
        for (int p = lo; p < hi; ++p) many.add(part[(size_t)p * d + e]);
        s = many.get();
    }
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && e < d) {
        float v[SUM_WARPS];
#pragma unroll
        for (int w = 0; w < SUM_WARPS; ++w) v[w] = sums[w][lane];
#pragma unroll
        for (int o = SUM_WARPS / 2; o; o >>= 1)
#pragma unroll
            for (int w = 0; w < o; ++w) v[w] += v[w + o];
        dgain[e] = more ? dgain[e] + v[0] : v[0];
    }
}

// Rows of up to 1024 elements a warp, up to 16384 a block, two chunks a thread while that is enough;
// threads 0: longer ones.
struct Shape {
    bool warp;
    int threads, ch, rows;  // of a block
};
constexpr Shape kLoop{false, LOOP_THREADS, 0, 1};
Shape shape_of(int d) {
    const int chunks = ceil_div(d, 8);
    if (chunks <= 128) return Shape{true, 128, chunks <= 32 ? 1 : chunks <= 64 ? 2 : 4, 4};
    const int ch = chunks <= 2 * MAX_THREADS ? 2 : 4, threads = ceil_div(ceil_div(chunks, ch), 32) * 32;
    return threads <= MAX_THREADS ? Shape{false, threads, ch, 1} : Shape{false, 0, 0, 1};
}
bool whole16(const void *p, long long stride, int es) { return !(((uintptr_t)p | (uintptr_t)(stride * es)) & 15); }

// Blocks that walk `n` rows, `per_sm` threads an SM: forward 99 us with 1024, 106 with 1536, 129 with 700
// (16384 x 5120); backward 49 with 640, 53 with 1024, 61 with 800.
int blocks_of(const Shape &s, long long n, int n_sm, int per_sm) {
    const long long all = ceil_div_ll(n, s.rows), held = (long long)n_sm * (per_sm / s.threads > 1 ? per_sm / s.threads : 1);
    return (int)(all < held ? all : held);
}
constexpr int FWD_THREADS = 1024, BACK_THREADS = 640;
constexpr int LEAST_RUN = 208;
template <typename T, bool WARP, int CH, bool E8>
cudaError_t run_norm(const NormArgs &a, const Shape &s, int n_sm, cudaStream_t st) {
    return launch_k(norm_kernel<T, WARP, CH, E8>, dim3(blocks_of(s, a.n, n_sm, FWD_THREADS)), dim3(s.threads), 0, st, a);
}
template <typename T, bool WARP, int CH>
cudaError_t run_back(const NormBackArgs &a, const Shape &s, int n_sm, cudaStream_t st) {
    return launch_k(norm_back_kernel<T, WARP, CH>, dim3(blocks_of(s, a.n, n_sm, BACK_THREADS)), dim3(s.threads), 0, st, a);
}
template <typename T>
cudaError_t run_back_loop(const NormBackArgs &a, int parts, cudaStream_t st) {
    return launch_k(norm_back_loop_kernel<T>, dim3(parts), dim3(LOOP_THREADS), 0, st, a);
}
template <typename T, bool E8>
cudaError_t norm_shapes(const NormArgs &a, const Shape &s, int n_sm, cudaStream_t st) {
    const auto run = s.warp ? s.ch == 1 ? run_norm<T, true, 1, E8> : s.ch == 2 ? run_norm<T, true, 2, E8> : run_norm<T, true, 4, E8>
                            : s.ch == 2 ? run_norm<T, false, 2, E8> : run_norm<T, false, 4, E8>;
    return run(a, s, n_sm, st);
}
template <typename T>
cudaError_t back_shapes(const NormBackArgs &a, const Shape &s, int n_sm, cudaStream_t st) {
    const auto run = s.warp ? s.ch == 1 ? run_back<T, true, 1> : s.ch == 2 ? run_back<T, true, 2> : run_back<T, true, 4>
                            : s.ch == 2 ? run_back<T, false, 2> : run_back<T, false, 4>;
    return run(a, s, n_sm, st);
}

}  // namespace

cudaError_t launch_norm(const NormArgs &a, int n_sm, cudaStream_t st) {
    const int es = a.dtype == SP_F32 ? 4 : 2;
    const bool e8 = a.out_dtype == SP_E4M3;
    const bool y_whole = e8 ? !(((uintptr_t)a.y | (uintptr_t)a.ys) & 7) : whole16(a.y, a.ys, es);
    const bool vec = a.d % 8 == 0 && whole16(a.x, a.xs, es) && (!a.r || whole16(a.r, a.rs, es)) &&
                     (!a.sum || whole16(a.sum, a.ss, es)) && y_whole && whole16(a.gain, 0, 4);
    const Shape s = shape_of(a.d);
    if (!vec || !s.threads) {
        if (a.dtype == SP_F32) return launch_k(norm_loop_kernel<float>, dim3(a.n), dim3(LOOP_THREADS), 0, st, a);
        return launch_k(norm_loop_kernel<bf16>, dim3(a.n), dim3(LOOP_THREADS), 0, st, a);
    }
    if (e8) return a.dtype == SP_F32 ? norm_shapes<float, true>(a, s, n_sm, st) : norm_shapes<bf16, true>(a, s, n_sm, st);
    return a.dtype == SP_F32 ? norm_shapes<float, false>(a, s, n_sm, st) : norm_shapes<bf16, false>(a, s, n_sm, st);
}

int norm_back_parts(int n, int d, int n_sm) {
    Shape s = shape_of(d);
    if (!s.threads) s = kLoop;
    const int held = blocks_of(s, n, n_sm, BACK_THREADS) * s.rows, loop = blocks_of(kLoop, n, n_sm, BACK_THREADS);
    return held > loop ? held : loop;  // (which kernel it is depends on the alignment)
}

cudaError_t launch_norm_backward(const NormBackArgs &a, int n_sm, cudaStream_t st) {
    const int es = a.dtype == SP_F32 ? 4 : 2;
    const bool vec = a.d % 8 == 0 && whole16(a.dx, a.xs, es) && (!a.ds || whole16(a.ds, a.rs, es)) &&
                     whole16(a.s, a.ss, es) && whole16(a.dy, a.ys, es) && whole16(a.gain, 0, 4);
    const Shape s = shape_of(a.d);
    const bool loop = !vec || !s.threads;
    const Shape &shape = loop ? kLoop : s;
    // The gain's gradient of many rows: as many at a time as leave a walker LEAST_RUN rows, or the root of its rows,
    // to add up in one number, so that no sum is long.  4000001 equal fp32 rows of 64, 1316 a walker: off by up to
    // 2.0e-5 in one sum, 2.7e-6 so; 2000000 of them 852 us in one launch, 919 in four, 200000 bf16 ones of 2560 815
    // and 828.  (Walkers that add what they have to their partial rows every 64 rows: 890 and 833, and 1541 instead of
    // 1473 for 40000 of 12288.)
    const long long walkers = (long long)blocks_of(shape, a.n, n_sm, BACK_THREADS) * shape.rows, rows = ceil_div_ll(a.n, walkers);
    long long times = 1;
    if (a.dgain) {
        long long run = LEAST_RUN;
        while (run * run < rows) ++run;
        times = ceil_div_ll(rows, run);
    }
    const long long per = ceil_div_ll(rows, times) * walkers;
    for (long long r0 = 0; r0 < a.n; r0 += per) {
        NormBackArgs p = a;
        const auto from = [&](const void *x, long long stride) { return x ? (const char *)x + r0 * stride * es : nullptr; };
        p.n = (int)(per < a.n - r0 ? per : a.n - r0);
        p.dy = from(a.dy, a.ys);
        p.s = from(a.s, a.ss);
        p.ds = from(a.ds, a.rs);
        p.dx = const_cast<char *>(from(a.dx, a.xs));
        const int parts = blocks_of(shape, p.n, n_sm, BACK_THREADS);
        cudaError_t e;
        if (loop) e = a.dtype == SP_F32 ? run_back_loop<float>(p, parts, st) : run_back_loop<bf16>(p, parts, st);
        else e = a.dtype == SP_F32 ? back_shapes<float>(p, s, n_sm, st) : back_shapes<bf16>(p, s, n_sm, st);
        if (e == cudaSuccess && a.dgain)
            e = launch_k(norm_gain_kernel, dim3(ceil_div(a.d, 32)), dim3(32 * SUM_WARPS), 0, st, (const float *)a.part,
                         parts * shape.rows, a.d, a.dgain, (int)(r0 > 0));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace sp

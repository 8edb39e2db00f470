// Rotary positions, appending to a token cache and reading it back (Sec. 3.3: the
// draft head's cache that the classify path reads).  All three move each byte once and
// compute little: HBM bounds the large calls, the launch the small ones.
#include "sp_cache.cuh"

namespace sp {

namespace {

constexpr int THREADS = 256;

template <typename T, int V>
__device__ __forceinline__ void loadv(const T *p, float (&v)[V]) {
    if constexpr (V == 8 && sizeof(T) == 2) {
        load8(p, v);
    } else if constexpr (V == 4 && sizeof(T) == 4) {
        const float4 f = *(const float4 *)p;
        v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = to_f(p[i]);
    }
}
template <typename T, int V>
__device__ __forceinline__ void storev(T *p, const float (&v)[V]) {
    if constexpr (V == 8 && sizeof(T) == 2) {
        *(uint4 *)p = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]),
                                 pack2_bf16(v[6], v[7]));
    } else if constexpr (V == 4 && sizeof(T) == 4) {
        *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = from_f<T>(v[i]);
    }
}

// Rotate (or turn back) heads.  A block takes a few tokens: it first forms the
// (cos, sin) of their pairs in shared memory (one sincospif a (token, pair), shared by
// all heads), then its threads walk the (token, head, vector) units; a unit reads the
// two vectors that turn into one another (half layout) or one vector of whole pairs
// (interleaved), or copies a vector of the dims that pass.  V elements a vector: 16
// bytes, or 1 (2 interleaved) where a stride, base or width does not allow that.
template <typename T, int V, bool INTER>
__global__ void __launch_bounds__(THREADS) rotate_kernel(const __grid_constant__ RotateArgs a) {
    extern __shared__ float2 cs[];  // [token][pair]
    pdl_wait();
    pdl_trigger();
    const int half = a.rot.half, t0 = blockIdx.x * a.tokens_per_block;
    const int nt = min(a.tokens_per_block, a.n_tokens - t0);
    for (int i = threadIdx.x; i < nt * half; i += THREADS) {
        const int t = i / half;
        float2 v = rotary_cs(a.rot, a.pos[t0 + t], i - t * half);
        if (a.backward) v.y = -v.y;
        cs[i] = v;
    }
    __syncthreads();
    const int turn = (INTER ? a.rot.rot : half) / V, units = turn + (a.dh - a.rot.rot) / V;
    const int per_token = a.n_heads * units;
    for (int u = threadIdx.x; u < nt * per_token; u += THREADS) {
        const int t = u / per_token, r = u - t * per_token, h = r / units, c = r - h * units;
        const T *x = (const T *)a.x + (t0 + t) * a.xt + h * a.xh;
        T *y = (T *)a.y + (t0 + t) * a.yt + h * a.yh;
        if (c >= turn) {
            const int e = a.rot.rot + (c - turn) * V;
            float v[V];
            loadv<T, V>(x + e, v);
            storev<T, V>(y + e, v);
        } else if constexpr (INTER) {
            float v[V];
            loadv<T, V>(x + c * V, v);
            const float2 *w = cs + t * half + c * (V / 2);
#pragma unroll
            for (int i = 0; i < V; i += 2) {
                const float2 k = w[i / 2];
                const float p = v[i], q = v[i + 1];
                v[i] = p * k.x - q * k.y;
                v[i + 1] = q * k.x + p * k.y;
            }
            storev<T, V>(y + c * V, v);
        } else {
            float p[V], q[V];
            loadv<T, V>(x + c * V, p);
            loadv<T, V>(x + half + c * V, q);
            const float2 *w = cs + t * half + c * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float2 k = w[i];
                const float s = p[i];
                p[i] = s * k.x - q[i] * k.y;
                q[i] = q[i] * k.x + s * k.y;
            }
            storev<T, V>(y + c * V, p);
            storev<T, V>(y + half + c * V, q);
        }
    }
}

template <typename T, int V>
cudaError_t run_rotate(const RotateArgs &a, cudaStream_t st) {
    const dim3 grid(ceil_div(a.n_tokens, a.tokens_per_block));
    const size_t smem = (size_t)a.tokens_per_block * a.rot.half * sizeof(float2);
    if (a.rot.interleaved) return launch_k(rotate_kernel<T, V == 1 ? 2 : V, true>, grid, dim3(THREADS), smem, st, a);
    return launch_k(rotate_kernel<T, V, false>, grid, dim3(THREADS), smem, st, a);
}

// 8 elements of a row, in vectors where the caller's rows allow them.
__device__ __forceinline__ void load_row8(const void *p, int dtype, long long e, int vec, float (&v)[8]) {
    if (dtype == SP_F32) {
        const float *s = (const float *)p + e;
        if (vec) {
            load8(s, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = s[i];
        }
    } else {
        const bf16 *s = (const bf16 *)p + e;
        if (vec) {
            load8(s, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = to_f(s[i]);
        }
    }
}
__device__ __forceinline__ void store_row8(void *p, int dtype, long long e, int vec, const float (&v)[8]) {
    if (dtype == SP_F32) {
        float *d = (float *)p + e;
        if (vec) {
            *(float4 *)d = make_float4(v[0], v[1], v[2], v[3]);
            *(float4 *)(d + 4) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = v[i];
        }
    } else {
        bf16 *d = (bf16 *)p + e;
        if (vec) {
            *(uint4 *)d = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]),
                                     pack2_bf16(v[6], v[7]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = __float2bfloat16_rn(v[i]);
        }
    }
}

// The tokens of batch entry b that a copy kernel's block works on.
struct Chunk {
    SeqRef sq;
    int b, count, row0, j0, n;
};
__device__ __forceinline__ Chunk chunk_of(const CopyArgs &a, int *status) {
    Chunk c;
    const int b = blockIdx.x / a.chunks;
    c.b = b;
    c.sq = resolve_seq(a.seq_ids, a.seq_lens, 0, b, a.cache.kv.n_seqs, a.cache.max_seq_len, status);
    c.count = a.rows.count ? a.rows.count[b] : a.rows.max_rows;
    if (c.count < 0 || c.count > a.rows.max_rows) {
        if (status) atomicOr(status, SP_DEV_BAD_ROW);
        c.count = c.count < 0 ? 0 : a.rows.max_rows;
    }
    c.row0 = a.rows.row0 ? a.rows.row0[b] : b * a.rows.max_rows;
    c.j0 = (blockIdx.x - b * a.chunks) * a.tokens_per_block;
    c.n = max(0, min(a.tokens_per_block, c.count - c.j0));
    return c;
}
__device__ __forceinline__ bool row_of(const CopyArgs &a, const Chunk &c, int j, bool take, long long *row) {
    *row = (long long)c.row0 + (take && a.rows.take ? a.rows.take[(size_t)c.b * a.rows.max_rows + j] : j);
    return *row >= 0 && *row < a.rows.n_rows;
}

// Append: a block takes a few tokens of one sequence, dh / 8 lanes a (token, K or V,
// head) row, eight elements a lane.  The row's amax is a shuffle among its lanes; the
// partner of a rotated element is read again (its line is in L1).
template <int LANES>
__global__ void __launch_bounds__(THREADS) append_kernel(const __grid_constant__ CopyArgs a) {
    extern __shared__ float2 cs[];  // [token][pair]
    pdl_wait();
    pdl_trigger();
    const Chunk ck = chunk_of(a, threadIdx.x == 0 && blockIdx.x % a.chunks == 0 ? a.status : nullptr);
    const CacheDev &c = a.cache;
    const int half = a.rot.half, Hkv = c.Hkv, dh = LANES * 8;
    for (int i = threadIdx.x; i < ck.n * half; i += THREADS) {
        const int t = i / half;
        cs[i] = rotary_cs(a.rot, ck.sq.len + ck.j0 + t, i - t * half);
    }
    __syncthreads();
    const int rows = ck.sq.sid < 0 ? 0 : ck.n * 2 * Hkv;  // rows of this block
    const int lane = threadIdx.x % LANES;
    int bad = 0;
    for (int r0 = threadIdx.x / LANES; r0 < ceil_div(rows, THREADS / LANES) * (THREADS / LANES); r0 += THREADS / LANES) {
        const bool in = r0 < rows;  // (whole warps stay for the shuffles)
        const int r = in ? r0 : 0, j = r / (2 * Hkv), rem = r - j * 2 * Hkv, is_v = rem / Hkv, h = rem - is_v * Hkv;
        const int t = ck.sq.len + ck.j0 + j;
        long long src = 0, dst = 0;
        int step = 0;
        bool ok = in;
        if (ok && t >= c.max_seq_len) ok = false, bad |= SP_DEV_BAD_LENGTH;
        if (ok && !row_of(a, ck, ck.j0 + j, true, &src)) ok = false, bad |= SP_DEV_BAD_ROW;
        if (ok && !cache_row(c, ck.sq.sid, t, &dst, &step)) ok = false, bad |= SP_DEV_BAD_PAGE;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        const long long e0 = src * (is_v ? a.rows.v_stride : a.rows.k_stride) + h * dh;
        const void *from = is_v ? a.v : a.k;
        const int e = lane * 8;
        if (ok) {
            load_row8(from, a.dtype, e0 + e, a.vec, v);
            if (!is_v && e < a.rot.rot) {
                const float2 *w = cs + j * half;
                if (a.rot.interleaved) {
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        if (e + i >= a.rot.rot) break;
                        const float2 k = w[(e + i) / 2];
                        const float p = v[i], q = v[i + 1];
                        v[i] = p * k.x - q * k.y;
                        v[i + 1] = q * k.x + p * k.y;
                    }
                } else if (half % 8 == 0) {
                    float o[8];
                    const bool lo = e < half;
                    load_row8(from, a.dtype, e0 + (lo ? e + half : e - half), a.vec, o);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 k = w[(lo ? e : e - half) + i];
                        v[i] = lo ? v[i] * k.x - o[i] * k.y : v[i] * k.x + o[i] * k.y;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (e + i >= a.rot.rot) break;
                        const bool lo = e + i < half;
                        const int pair = lo ? e + i : e + i - half;
                        const long long at = e0 + (lo ? e + i + half : pair);
                        const float o = a.dtype == SP_F32 ? ((const float *)from)[at] : to_f(((const bf16 *)from)[at]);
                        const float2 k = w[pair];
                        v[i] = lo ? v[i] * k.x - o * k.y : v[i] * k.x + o * k.y;
                    }
                }
            }
        }
        if (c.dtype == SP_E4M3) {
            float amax = kMinAmax;
#pragma unroll
            for (int i = 0; i < 8; ++i) amax = fmaxf(amax, isfinite(v[i]) ? fabsf(v[i]) : 0.f);
#pragma unroll
            for (int o = 1; o < LANES; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
            const float inv = kMaxCode / amax;
            if (ok) {
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)  // x - x: 0, or NaN for what is not finite
                    w[i] = float_to_codes2(v[2 * i] * inv + (v[2 * i] - v[2 * i]),
                                           v[2 * i + 1] * inv + (v[2 * i + 1] - v[2 * i + 1]));
                const long long row = dst + (long long)h * step;
                *(uint2 *)((uint8_t *)cache_base(c, ck.sq.sid, is_v) + row * dh + e) =
                    make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
                if (lane == 0) scale_base(c, ck.sq.sid, is_v)[row] = amax / kMaxCode;
            }
        } else if (ok) {
            store_row8(cache_base(c, ck.sq.sid, is_v), c.dtype, (dst + (long long)h * step) * dh + e, 1, v);
        }
    }
    if (bad && a.status) atomicOr(a.status, bad);
}

// Read back: the same units the other way; tokens outside the sequence give zeros.
template <int LANES>
__global__ void __launch_bounds__(THREADS) read_kernel(const __grid_constant__ CopyArgs a) {
    pdl_wait();
    pdl_trigger();
    const Chunk ck = chunk_of(a, threadIdx.x == 0 && blockIdx.x % a.chunks == 0 ? a.status : nullptr);
    const CacheDev &c = a.cache;
    const int Hkv = c.Hkv, dh = LANES * 8, rows = ck.n * 2 * Hkv, lane = threadIdx.x % LANES, e = lane * 8;
    const int first = a.first ? a.first[ck.b] : 0;
    int bad = 0;
#pragma unroll 2
    for (int r = threadIdx.x / LANES; r < rows; r += THREADS / LANES) {
        const int j = r / (2 * Hkv), rem = r - j * 2 * Hkv, is_v = rem / Hkv, h = rem - is_v * Hkv;
        long long dst, src;
        if (!row_of(a, ck, ck.j0 + j, false, &dst)) {
            bad |= SP_DEV_BAD_ROW;
            continue;
        }
        const int jj = a.rows.take ? a.rows.take[(size_t)ck.b * a.rows.max_rows + ck.j0 + j] : ck.j0 + j;
        const long long t = (long long)first + jj;
        int step;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (ck.sq.sid >= 0 && t >= 0 && t < ck.sq.len) {
            if (cache_row(c, ck.sq.sid, (int)t, &src, &step)) {
                src += (long long)h * step;
                const void *base = cache_base(c, ck.sq.sid, is_v);
                if (c.dtype == SP_E4M3) {
                    codes_to_float(*(const uint2 *)((const uint8_t *)base + src * dh + e), v);
                    const float s = scale_base(c, ck.sq.sid, is_v)[src];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= s;
                } else {
                    load_row8(base, c.dtype, src * dh + e, 1, v);
                }
            } else {
                bad |= SP_DEV_BAD_PAGE;
            }
        }
        store_row8(is_v ? a.v : a.k, a.dtype, dst * (is_v ? a.rows.v_stride : a.rows.k_stride) + h * dh + e, a.vec, v);
    }
    if (bad && a.status) atomicOr(a.status, bad);
}

// Tokens a block takes: several where that still leaves every SM a few blocks.
int tokens_a_block(long long tokens, int n_sm) {
    int t = 8;
    while (t > 1 && tokens < (long long)t * n_sm * 8) t >>= 1;
    return t;
}

}  // namespace

cudaError_t launch_rotate(int dtype, const RotateArgs &in, int n_sm, cudaStream_t st) {
    RotateArgs a = in;
    const int es = dtype == SP_F32 ? 4 : 2, V = 16 / es;
    const long long strides = a.xt | a.xh | a.yt | a.yh;
    const bool vec = !(((uintptr_t)a.x | (uintptr_t)a.y) & 15) && strides % V == 0 &&
                     (a.rot.interleaved ? a.rot.rot : a.rot.half) % V == 0 && (a.dh - a.rot.rot) % V == 0;
    a.tokens_per_block = tokens_a_block(a.n_tokens, n_sm);
    if (dtype == SP_F32) return vec ? run_rotate<float, 4>(a, st) : run_rotate<float, 1>(a, st);
    return vec ? run_rotate<bf16, 8>(a, st) : run_rotate<bf16, 1>(a, st);
}

cudaError_t launch_append(const CopyArgs &in, int n_sm, cudaStream_t st) {
    CopyArgs a = in;
    a.tokens_per_block = tokens_a_block((long long)a.B * a.rows.max_rows, n_sm);
    a.chunks = ceil_div(a.rows.max_rows, a.tokens_per_block);
    if ((long long)a.chunks * a.B > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    const dim3 grid(a.chunks * a.B);
    const size_t smem = (size_t)a.tokens_per_block * a.rot.half * sizeof(float2);
    if (a.cache.dh == 128) return launch_k(append_kernel<16>, grid, dim3(THREADS), smem, st, a);
    if (a.cache.dh == 64) return launch_k(append_kernel<8>, grid, dim3(THREADS), smem, st, a);
    return launch_k(append_kernel<4>, grid, dim3(THREADS), smem, st, a);
}

cudaError_t launch_read(const CopyArgs &in, int n_sm, cudaStream_t st) {
    CopyArgs a = in;
    a.tokens_per_block = tokens_a_block((long long)a.B * a.rows.max_rows, n_sm);
    a.chunks = ceil_div(a.rows.max_rows, a.tokens_per_block);
    if ((long long)a.chunks * a.B > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    const dim3 grid(a.chunks * a.B);
    if (a.cache.dh == 128) return launch_k(read_kernel<16>, grid, dim3(THREADS), 0, st, a);
    if (a.cache.dh == 64) return launch_k(read_kernel<8>, grid, dim3(THREADS), 0, st, a);
    return launch_k(read_kernel<4>, grid, dim3(THREADS), 0, st, a);
}

}  // namespace sp

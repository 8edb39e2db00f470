// Rotary positions, appending to a token cache and reading it back (Sec. 3.3: the
// draft head's cache that the classify path reads).  All three move each byte once and
// compute little: HBM bounds the large calls, the launch the small ones.
#include "sp_cache.cuh"

namespace sp {

namespace {

constexpr int THREADS = 256;
constexpr int GROUPS = 4;  // most token groups of a rotating block (16: the same)

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

// V elements as they lie: 16 bytes, or one by one, of which `left` exist.
template <typename T, int V>
struct RawVec {
    static constexpr bool WIDE = V * sizeof(T) == 16;
    union {
        uint4 w;
        T e[V];
    };
    __device__ __forceinline__ RawVec() {}
    __device__ __forceinline__ void load(const T *p, int left) {
        if constexpr (WIDE) {
            w = *(const uint4 *)p;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < left) e[i] = p[i];
        }
    }
    __device__ __forceinline__ void store(T *p, int left) const {
        if constexpr (WIDE) {
            *(uint4 *)p = w;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < left) p[i] = e[i];
        }
    }
    __device__ __forceinline__ void get(float (&v)[V]) const {
        if constexpr (V == 8) {
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(u[i] << 16), v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = to_f(e[i]);
        }
    }
};

// Rotate (or turn back) heads.  A thread has one unit of a head -- the two vectors that
// turn into one another (half layout), one vector of whole pairs (interleaved), or one
// vector of the dims that pass (a pair's scalar vector may have one element left) -- for every
// head it visits of a token, U heads at a time: the next ones' loads are under way, as they
// lie, while these are turned.  (cos, sin) of the block's tokens are formed in shared memory
// behind the first loads (one sincospif a (token, pair), shared by all heads).  V elements a
// vector: 16 bytes, or 1 (2 interleaved) where a stride, base or width does not allow that.  A
// group of tokens fills the block; a block takes up to GROUPS of them one after another.
// HBM-bound where large: 16384 tokens of 48 bf16 heads, half of each in pairs, 61 us, 6.6 TB/s
// (one group a block, hence nothing to load ahead: 69; values held as floats: 85); 4099 tokens of
// 40 fp32 heads turned back, one group a block, 27.3 us, 6.2 TB/s; 16 tokens 5.3 to 5.8 us (a
// launch).
template <typename T, int V, bool INTER>
__global__ void __launch_bounds__(THREADS, 4) rotate_kernel(const __grid_constant__ RotateArgs a) {
    extern __shared__ float2 cs[];  // [token][pair]
    constexpr int U = INTER ? 4 : 2, W = INTER ? V / 2 : V;  // heads in flight, pairs of a unit
    pdl_wait();
    pdl_trigger();
    const int half = a.rot.half, turn = (INTER ? a.rot.rot : half) / V, units = turn + ceil_div(a.dh - a.rot.rot, V);
    const int wide = min(units, THREADS), heads = min(a.n_heads, THREADS / wide), nt = a.tokens_per_block;
    const int per = wide * heads, tl = threadIdx.x / per, rest = threadIdx.x - tl * per, h0 = rest / wide;
    const int c0 = rest - h0 * wide, t0 = blockIdx.x * nt * a.groups, end = min(t0 + nt * a.groups, a.n_tokens);
    struct Vecs {
        RawVec<T, V> p[U], q[INTER ? 1 : U];
    };
    struct At {  // what a thread does next: heads h, h + heads .. of a unit of token t
        int t, c, h;
    };
    auto place = [&](int unit) { return unit < turn ? unit * V : a.rot.rot + (unit - turn) * V; };
    auto load = [&](At i, Vecs &v) {
        const T *x = (const T *)a.x + i.t * a.xt + i.h * a.xh + place(i.c);
        const long long step = heads * a.xh;
#pragma unroll
        for (int u = 0; u < U; ++u, x += step) {
            if (i.h + u * heads >= a.n_heads) break;
            v.p[u].load(x, a.dh - place(i.c));
            if constexpr (!INTER) {
                if (i.c < turn) v.q[u].load(x + half, V);
            }
        }
    };
    At at{tl < nt ? t0 + tl : end, c0, h0};
    Vecs v, ahead;
    if (at.t < end) load(at, v);
    for (int i = threadIdx.x; i < (end - t0) * half; i += THREADS) {
        const int k = i / half;
        float2 f = rotary_cs(a.rot, a.pos[t0 + k], i - k * half);
        if (a.backward) f.y = -f.y;
        cs[i] = f;
    }
    __syncthreads();
#pragma unroll 1
    while (at.t < end) {
        At next = at;
        next.h += U * heads;
        if (next.h >= a.n_heads) {
            next.h = h0;
            next.c += wide;
            if (next.c >= units) {
                next.c = c0;
                next.t += nt;
            }
        }
        if (next.t < end) load(next, ahead);
        T *y = (T *)a.y + at.t * a.yt + at.h * a.yh + place(at.c);
        const long long step = heads * a.yh;
        if (at.c < turn) {
            float2 k[W];
#pragma unroll
            for (int i = 0; i < W; ++i) k[i] = cs[(at.t - t0) * half + at.c * W + i];
#pragma unroll
            for (int u = 0; u < U; ++u, y += step) {
                if (at.h + u * heads >= a.n_heads) break;
                float p[V], q[INTER ? 1 : V];
                v.p[u].get(p);
                if constexpr (!INTER) v.q[u].get(q);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    float *one, *two;
                    if constexpr (INTER) one = &p[2 * i], two = &p[2 * i + 1];
                    else one = &p[i], two = &q[i];
                    const float f = *one;
                    *one = f * k[i].x - *two * k[i].y;
                    *two = *two * k[i].x + f * k[i].y;
                }
                if constexpr (!INTER) storev<T, V>(y + half, q);
                storev<T, V>(y, p);
            }
        } else {  // dims that pass
#pragma unroll
            for (int u = 0; u < U; ++u, y += step) {
                if (at.h + u * heads >= a.n_heads) break;
                v.p[u].store(y, a.dh - place(at.c));
            }
        }
        v = ahead;
        at = next;
    }
}

template <typename T, int V, bool INTER>
cudaError_t run_rotate(RotateArgs a, int n_sm, cudaStream_t st) {
    const int turn = (INTER ? a.rot.rot : a.rot.half) / V, units = turn + ceil_div(a.dh - a.rot.rot, V);
    const int wide = units < THREADS ? units : THREADS, fit = THREADS / wide;
    const int per = wide * (a.n_heads < fit ? a.n_heads : fit);
    a.tokens_per_block = THREADS / per;
    // Groups of such tokens a block: up to GROUPS as long as every SM has 16 blocks, four rounds of
    // four (with half as many 4099 tokens took 27.5 instead of 27.3 us, with a quarter 31.8).
    a.groups = 1;
    while (a.groups < GROUPS && (long long)a.groups * 2 * a.tokens_per_block * n_sm * 16 <= a.n_tokens &&
           a.groups * 2 * a.tokens_per_block * a.rot.half <= 4096)
        a.groups *= 2;
    const int tokens = a.tokens_per_block * a.groups;
    const dim3 grid(ceil_div(a.n_tokens, tokens));
    const size_t smem = (size_t)tokens * a.rot.half * sizeof(float2);  // (at most 32 KB)
    return launch_k(rotate_kernel<T, V, INTER>, grid, dim3(THREADS), smem, st, a);
}
template <typename T, int V>
cudaError_t pick_rotate(const RotateArgs &a, int n_sm, cudaStream_t st) {
    if (a.rot.interleaved) return run_rotate<T, V == 1 ? 2 : V, true>(a, n_sm, st);
    return run_rotate<T, V, false>(a, n_sm, st);
}

// 8 elements to a row, in vectors where the row allows them.
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

// 8 elements of a row as they are in memory, and as floats.
template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const void *p, long long e, int vec) {
        const float *s = (const float *)p + e;
        if (vec) {
            a = *(const float4 *)s, b = *(const float4 *)(s + 4);
        } else {
            a = make_float4(s[0], s[1], s[2], s[3]), b = make_float4(s[4], s[5], s[6], s[7]);
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
};
template <>
struct Raw8<bf16> {
    uint4 u;
    __device__ __forceinline__ void load(const void *p, long long e, int vec) {
        const uint16_t *s = (const uint16_t *)p + e;
        if (vec) {
            u = *(const uint4 *)s;
        } else {
            u = make_uint4(s[0] | (uint32_t)s[1] << 16, s[2] | (uint32_t)s[3] << 16, s[4] | (uint32_t)s[5] << 16,
                           s[6] | (uint32_t)s[7] << 16);
        }
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
// 16 elements of a cached row.
template <typename T>
struct Cached16 {
    static constexpr bool codes = false;
    Raw8<T> a, b;
    __device__ __forceinline__ void load(const void *base, const float *, long long row, int dh, int e0, int e1) {
        a.load(base, row * dh + e0, 1);
        b.load(base, row * dh + e1, 1);
    }
    __device__ __forceinline__ void get(float (&v0)[8], float (&v1)[8]) const { a.get(v0), b.get(v1); }
};
struct Code16 {  // codes and their row's scale
    static constexpr bool codes = true;
    uint2 a, b;
    float s;
    __device__ __forceinline__ void load(const void *base, const float *scale, long long row, int dh, int e0, int e1) {
        const uint8_t *p = (const uint8_t *)base + row * dh;
        a = *(const uint2 *)(p + e0), b = *(const uint2 *)(p + e1);
        s = scale[row];
    }
    __device__ __forceinline__ void get(float (&v0)[8], float (&v1)[8]) const {
        codes_to_float(a, v0);
        codes_to_float(b, v1);
#pragma unroll
        for (int i = 0; i < 8; ++i) v0[i] *= s, v1[i] *= s;
    }
};

// The tokens of a batch entry that a copy kernel's block works on.
struct Chunk {
    SeqRef sq;
    int b, count, j0, n;
    long long row0;
};
__device__ __forceinline__ Chunk chunk_of(const CopyArgs &a, int *status) {
    Chunk c;
    const int b = blockIdx.x / a.chunks;
    c.b = b;
    c.sq = resolve_seq(a.seq_ids, a.seq_lens, 0, b, a.cache.kv.n_seqs, a.cache.max_seq_len, status);
    c.count = a.rows.count ? a.rows.count[b] : a.rows.max_rows;
    c.row0 = a.rows.row0 ? a.rows.row0[b] : (long long)b * a.rows.max_rows;
    if (c.count < 0 || c.count > a.rows.max_rows) {
        if (status) atomicOr(status, SP_DEV_BAD_ROW);
        c.count = c.count < 0 ? 0 : a.rows.max_rows;
    }
    c.j0 = (blockIdx.x - b * a.chunks) * a.tokens_per_block;
    c.n = max(0, min(a.tokens_per_block, c.count - c.j0));
    return c;
}

constexpr int MAX_TOK = 16;  // tokens of a block (32: the long contexts below read in 72 instead of 68 us)

// The (token, K or V, head) rows of a block in order, a fixed step at a time.
struct RowWalk {
    int jv, h;                 // 2 token + (V), head
    int heads, step_jv, step_h;
    __device__ __forceinline__ RowWalk(int r, int step, int Hkv)
        : jv(r / Hkv), h(r - r / Hkv * Hkv), heads(Hkv), step_jv(step / Hkv), step_h(step - step / Hkv * Hkv) {}
    __device__ __forceinline__ int j() const { return jv >> 1; }
    __device__ __forceinline__ int is_v() const { return jv & 1; }
    __device__ __forceinline__ void next() {
        h += step_h;
        jv += step_jv;
        if (h >= heads) h -= heads, ++jv;
    }
};

// Append: a block takes a few tokens of one sequence, dh / 16 lanes a (token, K or V,
// head) row, two chunks of eight elements a lane: chunks that turn into one another (half
// layout), so that a rotation stays in its lane, else neighbours.  U rows' loads are in
// flight, the first of them issued before the block looks up its tokens' pages and forms
// their (cos, sin).  The row's amax is a shuffle among its lanes.  Bound by its
// instructions (about ten an element: rotation, amax, scale, conversion) and its loads' latency:
// 12 prompts of 500 to 4000 tokens, 8 kv heads, rotated and quantised at 3.2 to 4.0 TB/s, 42 to
// 55 us by the lengths drawn (into bf16 pages, less to compute and more to write, 47 where 8 bits
// take 50: 5.0 TB/s); 64 accepted paths of up to 6 tokens in 4.7 us (a launch).  Three
// blocks an SM took 52 to 55 us, one row in flight 75 to 85.  (fp32 rows hold twice the
// registers: two blocks.)
template <typename T>
constexpr int kAppendBlocks = 2;  // blocks an SM
template <>
constexpr int kAppendBlocks<bf16> = 4;
template <int LANES, typename T>
__global__ void __launch_bounds__(THREADS, kAppendBlocks<T>) append_kernel(const __grid_constant__ CopyArgs a) {
    extern __shared__ float2 cs[];  // [token][pair]
    __shared__ long long place[MAX_TOK];  // the cache's (token, head 0) row; -1: skipped
    constexpr int U = 2, G = THREADS / LANES;  // rows in flight, rows of a pass
    pdl_wait();
    pdl_trigger();
    const Chunk ck = chunk_of(a, threadIdx.x == 0 && blockIdx.x % a.chunks == 0 ? a.status : nullptr);
    if (ck.n == 0 || ck.sq.sid < 0) return;  // uniform over the block
    const CacheDev &c = a.cache;
    const int half = a.rot.half, Hkv = c.Hkv, dh = LANES * 16;
    const int rows = ck.n * 2 * Hkv, lane = threadIdx.x % LANES, first = threadIdx.x / LANES;
    const int passes = ceil_div(rows, G);
    // this lane's two chunks
    const bool in_lane = !a.rot.interleaved && half % 8 == 0;  // (0 without a rotation)
    const int nh = in_lane ? half / 8 : 0;
    const int e0 = 8 * (lane < nh ? lane : 2 * lane), e1 = 8 * (lane < nh ? lane + nh : 2 * lane + 1);
    Raw8<T> x0[U], x1[U];
    auto source = [&](int j, int is_v, int h) {  // the row's first element; -1: none
        const long long row = ck.row0 + (a.rows.take ? a.rows.take[(size_t)ck.b * a.rows.max_rows + ck.j0 + j] : ck.j0 + j);
        return row >= 0 && row < a.rows.n_rows ? row * (is_v ? a.rows.v_stride : a.rows.k_stride) + h * dh : -1;
    };
    auto load = [&](RowWalk w, int pass) {
#pragma unroll
        for (int u = 0; u < U; ++u, w.next()) {
            if (first + (pass + u) * G >= rows) continue;
            const long long at = source(w.j(), w.is_v(), w.h);
            if (at < 0) continue;
            x0[u].load(w.is_v() ? a.v : a.k, at + e0, a.vec);
            x1[u].load(w.is_v() ? a.v : a.k, at + e1, a.vec);
        }
    };
    RowWalk w(first, G, Hkv);
    load(w, 0);
    if ((int)threadIdx.x < ck.n) {
        const int j = threadIdx.x;
        const long long t = (long long)ck.sq.len + ck.j0 + j;  // (a length near max_seq_len's own limit passes 31 bits)
        long long dst = -1;
        int bad = 0, step;
        // (a negative length reads as 0 above: its tokens would take the places of the first ones)
        if (t >= c.max_seq_len || a.seq_lens[ck.sq.sid] < 0) bad = SP_DEV_BAD_LENGTH;
        else if (source(j, 0, 0) < 0) bad = SP_DEV_BAD_ROW;
        else if (!cache_row(c, ck.sq.sid, (int)t, &dst, &step)) bad = SP_DEV_BAD_PAGE;
        place[j] = bad ? -1 : dst;
        if (bad && a.status) atomicOr(a.status, bad);
    }
    for (int i = threadIdx.x; i < ck.n * half; i += THREADS) {
        const int t = i / half;
        // (a position that wraps is past max_seq_len: its token is skipped)
        cs[i] = rotary_cs(a.rot, (int)((unsigned)ck.sq.len + ck.j0 + t), i - t * half);
    }
    __syncthreads();
    const int head_step = c.kv.layout == SP_KV_PAGED ? c.kv.page_size : 1;
    void *kb = cache_base(c, ck.sq.sid, 0), *vb = cache_base(c, ck.sq.sid, 1);
    float *ks = nullptr, *vs = nullptr;
    if (c.dtype == SP_E4M3) ks = scale_base(c, ck.sq.sid, 0), vs = scale_base(c, ck.sq.sid, 1);
#pragma unroll 1
    for (int pass = 0; pass < passes; pass += U) {
        if (pass > 0) load(w, pass);
#pragma unroll
        for (int u = 0; u < U; ++u, w.next()) {
            if (pass + u >= passes) break;  // (whole warps stay for the shuffles)
            const long long p0 = first + (pass + u) * G < rows ? place[w.j()] : -1;
            const bool ok = p0 >= 0;
            const long long dst = p0 + (long long)w.h * head_step;
            float v0[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, v1[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (ok) x0[u].get(v0), x1[u].get(v1);
            if (ok && half && !w.is_v()) {
                const float2 *k = cs + w.j() * half;
                if (in_lane) {
                    if (lane < nh) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float2 f = k[e0 + i];
                            const float p = v0[i];
                            v0[i] = p * f.x - v1[i] * f.y;
                            v1[i] = v1[i] * f.x + p * f.y;
                        }
                    }
                } else if (a.rot.interleaved) {
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        if (e0 + i >= a.rot.rot) break;  // (chunks 2 l and 2 l + 1)
                        const float2 f = k[e0 / 2 + i / 2];
                        float &one = i < 8 ? v0[i & 7] : v1[i & 7], &two = i < 8 ? v0[(i & 7) + 1] : v1[(i & 7) + 1];
                        const float p = one;
                        one = p * f.x - two * f.y;
                        two = two * f.x + p * f.y;
                    }
                } else {  // pairs across lanes: the partner is read from the row
                    const long long at = source(w.j(), 0, w.h);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (e0 + i >= a.rot.rot) break;
                        const bool one = e0 + i < half;
                        const int pair = one ? e0 + i : e0 + i - half;
                        const float z = to_f(((const T *)a.k)[at + (one ? e0 + i + half : pair)]);
                        const float2 f = k[pair];
                        float &y = i < 8 ? v0[i & 7] : v1[i & 7];
                        y = one ? y * f.x - z * f.y : y * f.x + z * f.y;
                    }
                }
            }
            if (c.dtype == SP_E4M3) {
                float amax = kMinAmax;
#pragma unroll
                for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fmaxf(fabsf(v0[i]), fabsf(v1[i])));  // (a NaN is no maximum)
#pragma unroll
                for (int q = 1; q < LANES; q <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, q));
                if (__any_sync(0xffffffffu, amax == INFINITY)) {  // rare: infinities do not set the scale, and become NaN
                    amax = kMinAmax;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        v0[i] += v0[i] - v0[i];
                        v1[i] += v1[i] - v1[i];
                        amax = fmaxf(amax, fmaxf(fabsf(v0[i]), fabsf(v1[i])));
                    }
#pragma unroll
                    for (int q = 1; q < LANES; q <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, q));
                }
                if (ok) {
                    const float inv = kMaxCode / amax;
                    auto codes = [&](const float(&v)[8]) {
                        return make_uint2(float_to_codes2(v[0] * inv, v[1] * inv) | float_to_codes2(v[2] * inv, v[3] * inv) << 16,
                                          float_to_codes2(v[4] * inv, v[5] * inv) | float_to_codes2(v[6] * inv, v[7] * inv) << 16);
                    };
                    uint8_t *to = (uint8_t *)(w.is_v() ? vb : kb) + dst * dh;
                    *(uint2 *)(to + e0) = codes(v0);
                    *(uint2 *)(to + e1) = codes(v1);
                    // (a product with a constant: the quotient took 62.7 instead of 55.3 us on the prompts above)
                    if (lane == 0) (w.is_v() ? vs : ks)[dst] = amax * (1.f / kMaxCode);
                }
            } else if (ok) {
                store_row8(w.is_v() ? vb : kb, c.dtype, dst * dh + e0, 1, v0);
                store_row8(w.is_v() ? vb : kb, c.dtype, dst * dh + e1, 1, v1);
            }
        }
    }
}

// Read back: rows the other way, 16 elements a lane; tokens outside the sequence give
// zeros.  A block's tokens are looked up once, then U rows a thread are in flight.  CT: the
// cache's elements (Code16: 8 bits).  Bound by its loads' latency and HBM: 6 contexts of 3000
// to 9000 tokens, 8 kv heads, 8-bit, as bf16 in 58 to 62 us, 5 TB/s (from bf16 pages 67 us, 5.7
// TB/s, from contiguous bf16 62); 3 of 100 to 700 tokens as fp32 in 7.2 us.  Sixteen neighbouring
// elements a lane, whose halves are stored 32 bytes apart, took 65 and 7.9 us, five blocks an SM
// 56 and 8.2, the next rows' loads under way 71 and 8.3.
template <int LANES, typename CT>
__global__ void __launch_bounds__(THREADS) read_kernel(const __grid_constant__ CopyArgs a) {
    __shared__ long long out_row[MAX_TOK], place[MAX_TOK];
    constexpr int U = 2, G = THREADS / LANES;  // rows in flight, rows of a pass
    pdl_wait();
    pdl_trigger();
    const Chunk ck = chunk_of(a, threadIdx.x == 0 && blockIdx.x % a.chunks == 0 ? a.status : nullptr);
    if (ck.n == 0) return;  // uniform over the block
    const CacheDev &c = a.cache;
    const int Hkv = c.Hkv, dh = LANES * 16, rows = ck.n * 2 * Hkv;
    const int e0 = threadIdx.x % LANES * 8, e1 = e0 + dh / 2;  // two chunks: neighbours store side by side
    const int head_step = c.kv.layout == SP_KV_PAGED ? c.kv.page_size : 1, sid = ck.sq.sid;
    if ((int)threadIdx.x < ck.n) {
        const int j = ck.j0 + threadIdx.x;
        const long long t = (a.first ? a.first[ck.b] : 0) +
                            (long long)(a.rows.take ? a.rows.take[(size_t)ck.b * a.rows.max_rows + j] : j);
        long long dst = ck.row0 + j, src = -1;
        int bad = 0, step;
        if (dst < 0 || dst >= a.rows.n_rows) bad = SP_DEV_BAD_ROW, dst = -1;
        else if (sid >= 0 && t >= 0 && t < ck.sq.len && !cache_row(c, sid, (int)t, &src, &step)) bad = SP_DEV_BAD_PAGE, src = -1;
        out_row[threadIdx.x] = dst;
        place[threadIdx.x] = src;
        if (bad && a.status) atomicOr(a.status, bad);
    }
    const void *kb = nullptr, *vb = nullptr;
    const float *ks = nullptr, *vs = nullptr;
    if (sid >= 0) {
        kb = cache_base(c, sid, 0), vb = cache_base(c, sid, 1);
        if constexpr (CT::codes) ks = scale_base(c, sid, 0), vs = scale_base(c, sid, 1);
    }
    __syncthreads();
    RowWalk w(threadIdx.x / LANES, G, Hkv);
#pragma unroll 1
    for (int r = threadIdx.x / LANES; r < rows; r += U * G) {
        CT x[U];
        RowWalk s = w;
#pragma unroll
        for (int u = 0; u < U; ++u, s.next()) {
            const long long p0 = r + u * G < rows ? place[s.j()] : -1;
            if (p0 < 0) continue;
            x[u].load(s.is_v() ? vb : kb, s.is_v() ? vs : ks, p0 + (long long)s.h * head_step, dh, e0, e1);
        }
#pragma unroll
        for (int u = 0; u < U; ++u, w.next()) {
            const long long row = r + u * G < rows ? out_row[w.j()] : -1;
            if (row < 0) continue;
            float v0[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, v1[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (place[w.j()] >= 0) x[u].get(v0, v1);
            const long long to = row * (w.is_v() ? a.rows.v_stride : a.rows.k_stride) + w.h * dh;
            store_row8(w.is_v() ? a.v : a.k, a.dtype, to + e0, a.vec, v0);
            store_row8(w.is_v() ? a.v : a.k, a.dtype, to + e1, a.vec, v1);
        }
    }
}

template <int LANES>
cudaError_t run_append(const CopyArgs &a, dim3 grid, cudaStream_t st) {
    const size_t smem = (size_t)a.tokens_per_block * a.rot.half * sizeof(float2);
    if (a.dtype == SP_F32) return launch_k(append_kernel<LANES, float>, grid, dim3(THREADS), smem, st, a);
    return launch_k(append_kernel<LANES, bf16>, grid, dim3(THREADS), smem, st, a);
}
template <int LANES>
cudaError_t run_read(const CopyArgs &a, dim3 grid, cudaStream_t st) {
    if (a.cache.dtype == SP_E4M3) return launch_k(read_kernel<LANES, Code16>, grid, dim3(THREADS), 0, st, a);
    if (a.cache.dtype == SP_F32) return launch_k(read_kernel<LANES, Cached16<float>>, grid, dim3(THREADS), 0, st, a);
    return launch_k(read_kernel<LANES, Cached16<bf16>>, grid, dim3(THREADS), 0, st, a);
}

// Tokens a block takes: as many as leave every SM two blocks (a block looks them up first; six
// blocks: three short contexts read in 8.7 instead of 8.3 us, the long ones as before).
int tokens_a_block(long long tokens, int n_sm) {
    int t = MAX_TOK;
    while (t > 1 && tokens < (long long)t * n_sm * 2) t >>= 1;
    return t;
}

}  // namespace

cudaError_t launch_rotate(int dtype, const RotateArgs &a, int n_sm, cudaStream_t st) {
    const int es = dtype == SP_F32 ? 4 : 2, V = 16 / es;
    const long long strides = a.xt | a.xh | a.yt | a.yh;
    const bool vec = !(((uintptr_t)a.x | (uintptr_t)a.y) & 15) && strides % V == 0 &&
                     (a.rot.interleaved ? a.rot.rot : a.rot.half) % V == 0 && (a.dh - a.rot.rot) % V == 0;
    if (dtype == SP_F32) return vec ? pick_rotate<float, 4>(a, n_sm, st) : pick_rotate<float, 1>(a, n_sm, st);
    return vec ? pick_rotate<bf16, 8>(a, n_sm, st) : pick_rotate<bf16, 1>(a, n_sm, st);
}

cudaError_t launch_append(const CopyArgs &in, int n_sm, cudaStream_t st) {
    CopyArgs a = in;
    a.tokens_per_block = tokens_a_block((long long)a.B * a.rows.max_rows, n_sm);
    a.chunks = ceil_div(a.rows.max_rows, a.tokens_per_block);
    if ((long long)a.chunks * a.B > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    const dim3 grid(a.chunks * a.B);
    if (a.cache.dh == 128) return run_append<8>(a, grid, st);
    if (a.cache.dh == 64) return run_append<4>(a, grid, st);
    return run_append<2>(a, grid, st);
}

cudaError_t launch_read(const CopyArgs &in, int n_sm, cudaStream_t st) {
    CopyArgs a = in;
    a.tokens_per_block = tokens_a_block((long long)a.B * a.rows.max_rows, n_sm);
    a.chunks = ceil_div(a.rows.max_rows, a.tokens_per_block);
    if ((long long)a.chunks * a.B > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    const dim3 grid(a.chunks * a.B);
    if (a.cache.dh == 128) return run_read<8>(a, grid, st);
    if (a.cache.dh == 64) return run_read<4>(a, grid, st);
    return run_read<2>(a, grid, st);
}

}  // namespace sp

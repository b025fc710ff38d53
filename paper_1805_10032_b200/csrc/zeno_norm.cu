// Layer norm of rows of activations, and its backward pass with the weight gradients reduced per group (worker).
//
// Bound by the activations' bytes: forward x in, y out; backward dy and x in, dx out, each once.  Forward: a row's entries stay in
// the registers of the 32 to 1024 threads that share it, between the sum, the centred squares and the result.  Backward: a
// thread owns columns, not rows: it goes down a stretch of a group's rows with the sums of its columns' weight gradients in
// registers, and copies of the rows ahead are in flight while a row's two averages are formed across the block.
#include "zeno_operators.h"
#include "zeno_saved.cuh"

namespace zeno {

namespace {

constexpr int kThreads = 256;

// Sum over a row's entries j of a block's thread
template <typename F>
__device__ __forceinline__ float sum_of_row(int64_t cols, F term) {
    LongSum s;
    for (int64_t j = threadIdx.x; j < cols;) {
        const int64_t end = min(cols, j + kShortSum * kThreads);
        float part = 0.f;
        for (; j < end; j += kThreads) part += term(j);
        s.add(part);
    }
    return s.sum;
}

// Rows of any length and alignment, a block each: the sum, then the centred squares, then the result, reading the row three
// times (twice of it from L1 or L2).
template <typename T, typename P>
__global__ void __launch_bounds__(kThreads) norm_any_kernel(NormArgs a) {
    __shared__ float scratch[2][kThreads / 32];
    const int64_t r = blockIdx.x;
    const T *x = static_cast<const T *>(a.x.data) + a.x.at(r);
    T *y = static_cast<T *>(a.y.data) + a.y.at(r);
    const P *w = static_cast<const P *>(a.w) + r / a.n * a.ldw;
    const P *b = a.b ? static_cast<const P *>(a.b) + r / a.n * a.ldw : nullptr;
    float s = sum_of_row(a.cols, [&](int64_t j) { return value_of(x + j); });
    const float mean = block_sum<kThreads>(s, scratch[0]) / (float)a.cols;
    s = sum_of_row(a.cols, [&](int64_t j) {
        const float d = value_of(x + j) - mean;
        return d * d;
    });
    const float rstd = rsqrtf(block_sum<kThreads>(s, scratch[1]) / (float)a.cols + a.eps);
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads)
        put(y + j, fmaf((value_of(x + j) - mean) * rstd, value_of(w + j), b ? value_of(b + j) : 0.f));
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
}

// The layer's input in the backward pass: an entry of a row as it was, or as it was kept in 8 bits.
template <typename T>
struct InputRow {
    const T *x;
    const uint8_t *codes;
    const float *scales;
    __device__ __forceinline__ InputRow(const NormGradArgs &a, int64_t r)
        : x(a.x.data ? static_cast<const T *>(a.x.data) + a.x.at(r) : nullptr),
          codes(a.x.data ? nullptr : static_cast<const uint8_t *>(a.codes.data) + a.codes.at(r)),
          scales(a.x.data ? nullptr : static_cast<const float *>(a.scales.data) + a.scales.at(r)) {}
    __device__ __forceinline__ float operator()(int64_t j) const {
        return x ? value_of(x + j) : saved_value(codes[j], scales[j / ZENO_SAVED_BLOCK]);
    }
};

template <typename T, typename P>
__global__ void __launch_bounds__(kThreads) norm_dx_any_kernel(NormGradArgs a) {
    __shared__ float scratch[2][kThreads / 32];
    const int64_t r = blockIdx.x;
    const T *dy = static_cast<const T *>(a.dy.data) + a.dy.at(r);
    T *dx = static_cast<T *>(a.dx.data) + a.dx.at(r);
    const P *w = static_cast<const P *>(a.w) + r / a.n * a.ldw;
    const InputRow<T> x(a, r);
    const float mean = a.mean[r], rstd = a.rstd[r];
    LongSum s1, s2;
    for (int64_t j = threadIdx.x; j < a.cols;) {
        const int64_t end = min(a.cols, j + kShortSum * kThreads);
        float p1 = 0.f, p2 = 0.f;
#pragma unroll 4
        for (; j < end; j += kThreads) {
            const float g = value_of(dy + j) * value_of(w + j);
            p1 += g;
            p2 = fmaf(g, (x(j) - mean) * rstd, p2);
        }
        s1.add(p1);
        s2.add(p2);
    }
    const float c1 = block_sum<kThreads>(s1.sum, scratch[0]) / (float)a.cols, c2 = block_sum<kThreads>(s2.sum, scratch[1]) / (float)a.cols;
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
        const float g = value_of(dy + j) * value_of(w + j), h = (x(j) - mean) * rstd;
        put(dx + j, rstd * (g - c1 - h * c2));
    }
}

// ---- rows in registers

// N consecutive entries that one load takes, as they lie in memory: 16 bytes, or a single one for rows of any alignment.
template <typename T, int N> struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Pack { T v[N]; };
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T *p) {
    Pack<T, N> r;
    if constexpr (N * sizeof(T) == 16) *reinterpret_cast<uint4 *>(&r) = *reinterpret_cast<const uint4 *>(p);
    else if constexpr (N * sizeof(T) == 32) {
        reinterpret_cast<uint4 *>(&r)[0] = reinterpret_cast<const uint4 *>(p)[0];
        reinterpret_cast<uint4 *>(&r)[1] = reinterpret_cast<const uint4 *>(p)[1];
    } else if constexpr (N * sizeof(T) == 8) *reinterpret_cast<uint2 *>(&r) = *reinterpret_cast<const uint2 *>(p);
    else if constexpr (N * sizeof(T) == 4) *reinterpret_cast<uint32_t *>(&r) = *reinterpret_cast<const uint32_t *>(p);
    else {
#pragma unroll
        for (int i = 0; i < N; ++i) r.v[i] = p[i];
    }
    return r;
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T *p, const float (&f)[N]) {
    Pack<T, N> r;
#pragma unroll
    for (int i = 0; i < N; ++i) put(r.v + i, f[i]);
    if constexpr (N * sizeof(T) == 16) *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<uint4 *>(&r);
    else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = r.v[i];
    }
}
template <typename T, int N>
__device__ __forceinline__ void values(const Pack<T, N> &r, float (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = value_of(r.v + i);
}

// N weights; WV: their alignment allows one load
template <bool WV, typename P, int N>
__device__ __forceinline__ void weights(const P *p, float (&f)[N]) {
    if constexpr (WV) values(load_pack<P, N>(p), f);
    else {
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = value_of(p + k);
    }
}

// The sum over the TPR threads of a row; rows of more than a warp own the block.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *scratch) {
    if constexpr (TPR == 32) return warp_sum(v);
    else return block_sum<TPR>(v, scratch);
}

// threads in a block of one-warp rows
constexpr int kRowBlock = 128;

// A row in TPR threads, NV packs of N entries each.  WV: the weights can be loaded N at a time too.  (Few rows: one token of 4096 bfloat16 takes
// 6 us, all of it the latency of two loads and two sums over the block.)
template <typename T, typename P, int N, int TPR, int NV, bool WV>
__global__ void __launch_bounds__(TPR == 32 ? kRowBlock : TPR) norm_row_kernel(NormArgs a, int64_t rows) {
    __shared__ float scratch[2][32];
    constexpr int kRows = TPR == 32 ? kRowBlock / 32 : 1;
    const int64_t r = (int64_t)blockIdx.x * kRows + (TPR == 32 ? threadIdx.x >> 5 : 0);
    const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x;
    if (r >= rows) return;                     // a whole warp's row
    const T *x = static_cast<const T *>(a.x.data) + a.x.at(r);
    T *y = static_cast<T *>(a.y.data) + a.y.at(r);
    const int cols = (int)a.cols, packs = cols / N;
    Pack<T, N> raw[NV];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * TPR < packs) raw[i] = load_pack<T, N>(x + (int64_t)(t + i * TPR) * N);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * TPR < packs) {
            float f[N];
            values(raw[i], f);
#pragma unroll
            for (int k = 0; k < N; ++k) s += f[k];
        }
    const float mean = row_sum<TPR>(s, scratch[0]) / (float)cols;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * TPR < packs) {
            float f[N];
            values(raw[i], f);
#pragma unroll
            for (int k = 0; k < N; ++k) s = fmaf(f[k] - mean, f[k] - mean, s);
        }
    const float rstd = rsqrtf(row_sum<TPR>(s, scratch[1]) / (float)cols + a.eps);
    const int64_t group = a.ldw ? r / a.n * a.ldw : 0;
    const P *w = static_cast<const P *>(a.w) + group;
    const P *b = a.b ? static_cast<const P *>(a.b) + group : nullptr;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * TPR < packs) {
            const int j = (t + i * TPR) * N;
            float f[N], wf[N], bf[N];
            values(raw[i], f);
            weights<WV>(w + j, wf);
#pragma unroll
            for (int k = 0; k < N; ++k) bf[k] = 0.f;
            if (b) weights<WV>(b + j, bf);
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = fmaf((f[k] - mean) * rstd, wf[k], bf[k]);
            store_pack<T, N>(y + j, f);
        }
    if (t == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
}

// The layer's input, N entries at a time: as it was, or codes and their block's scale
template <typename T, int N, bool SAVED> struct InputPack {
    Pack<T, N> x;
    __device__ __forceinline__ void load(const NormGradArgs &a, int64_t r, int j) { x = load_pack<T, N>(static_cast<const T *>(a.x.data) + a.x.at(r) + j); }
    __device__ __forceinline__ void get(float (&f)[N]) const { values(x, f); }
};
template <typename T, int N> struct InputPack<T, N, true> {
    Pack<uint8_t, N> codes;
    float scale;
    __device__ __forceinline__ void load(const NormGradArgs &a, int64_t r, int j) {
        codes = load_pack<uint8_t, N>(static_cast<const uint8_t *>(a.codes.data) + a.codes.at(r) + j);
        scale = (static_cast<const float *>(a.scales.data) + a.scales.at(r))[j / ZENO_SAVED_BLOCK];
    }
    __device__ __forceinline__ void get(float (&f)[N]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = saved_value(codes.v[i], scale);
    }
};

// dx of a row in TPR threads' registers: rows too long for the kernels by columns below, which give both gradients from one reading
// (20 x 1024 x 16384 bfloat16, weight gradients included: 884 us, 2.3 TB/s).
template <typename T, typename P, int N, int TPR, int NV, bool SAVED, bool WV>
__global__ void __launch_bounds__(TPR, TPR <= 512 ? 2 : 1) norm_dx_row_kernel(NormGradArgs a) {
    __shared__ float scratch[2][32];
    const int64_t r = blockIdx.x;
    const int t = threadIdx.x, cols = (int)a.cols, packs = cols / N;
    const T *dy = static_cast<const T *>(a.dy.data) + a.dy.at(r);
    T *dx = static_cast<T *>(a.dx.data) + a.dx.at(r);
    const P *w = static_cast<const P *>(a.w) + (a.ldw ? r / a.n * a.ldw : 0);
    const float mean = a.mean[r], rstd = a.rstd[r];
    Pack<T, N> d[NV];
    InputPack<T, N, SAVED> x[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * TPR < packs) {
            d[i] = load_pack<T, N>(dy + (int64_t)(t + i * TPR) * N);
            x[i].load(a, r, (t + i * TPR) * N);
        }
    float c1 = 0.f, c2 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * TPR < packs) {
            float g[N], h[N], wf[N];
            values(d[i], g);
            x[i].get(h);
            weights<WV>(w + (t + i * TPR) * N, wf);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                g[k] *= wf[k];
                c1 += g[k];
                c2 = fmaf(g[k], (h[k] - mean) * rstd, c2);
            }
        }
    c1 = block_sum<TPR>(c1, scratch[0]) / (float)cols;
    c2 = block_sum<TPR>(c2, scratch[1]) / (float)cols;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * TPR < packs) {
            float g[N], h[N], wf[N];
            values(d[i], g);
            x[i].get(h);
            weights<WV>(w + (t + i * TPR) * N, wf);
#pragma unroll
            for (int k = 0; k < N; ++k) g[k] = rstd * (g[k] * wf[k] - c1 - (h[k] - mean) * rstd * c2);
            store_pack<T, N>(dx + (int64_t)(t + i * TPR) * N, g);
        }
}

// ---- backward, by columns

// 16 bytes of activations as pairs
__device__ __forceinline__ void pairs(uint4 u, Two (&f)[2], float) {
    f[0] = Two{__uint_as_float(u.x), __uint_as_float(u.y)};
    f[1] = Two{__uint_as_float(u.z), __uint_as_float(u.w)};
}
__device__ __forceinline__ void pairs(uint4 u, Two (&f)[4], __nv_bfloat16) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = Two{__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)};
}
__device__ __forceinline__ uint4 from_pairs(const Two (&f)[2], float) {
    return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
}
__device__ __forceinline__ uint32_t bf16_pair(Two f) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint4 from_pairs(const Two (&f)[4], __nv_bfloat16) { return make_uint4(bf16_pair(f[0]), bf16_pair(f[1]), bf16_pair(f[2]), bf16_pair(f[3])); }

// Rows of whole vectors.  A block: ROWS rows side by side, TPR threads each with NV = 2 vectors of columns, down the rows [first, last) of
// group blockIdx.y.  A thread stages its own columns of the rows ahead in shared memory by asynchronous copies that nobody
// else reads, so they need no registers and no barrier; the one barrier a row is that of its two averages.  (20 x 2048 x 4096 bfloat16: 173 us, 5.8 TB/s
// of what has to move; with the rows ahead in registers and a number to an instruction 480 us, bound by instructions.)  Then the sums of the
// ROWS rows' threads are joined, and go to the group's gradients, or (several blocks to a group) to `part` [group][block][dw, db][cols].
constexpr int kNV = 2;
template <typename T, bool SAVED> constexpr int kSlotBytes = 16 + (SAVED ? 16 / (int)sizeof(T) : 16);     // a vector of dy, and of x or its codes

template <typename T, typename P, int TPR, int ROWS, int STAGES, bool SAVED, bool DX>
__global__ void __launch_bounds__(TPR *ROWS, TPR *ROWS <= 256 ? 2 : 1) norm_columns_kernel(NormGradArgs a, float *part) {
    constexpr int N = 16 / sizeof(T), H = N / 2, kWarps = TPR / 32, kThreadsHere = TPR * ROWS;
    constexpr int kXBytes = SAVED ? N : 16;
    extern __shared__ __align__(16) uint8_t ring[];            // [STAGES][NV][threads] vectors of dy, then the same of x, then (SAVED) of scales
    __shared__ __align__(16) float2 scratch[2][ROWS][kWarps];
    uint8_t *ring_x = ring + STAGES * kNV * kThreadsHere * 16;
    float *ring_s = reinterpret_cast<float *>(ring_x + STAGES * kNV * kThreadsHere * kXBytes);
    const int tid = threadIdx.x, sub = tid / TPR, t = tid % TPR;
    const int cols = (int)a.cols, chunks = gridDim.x, i = blockIdx.y;
    const int64_t first = a.n * blockIdx.x / chunks + sub, last = a.n * (blockIdx.x + 1) / chunks;
    const float inv = 1.f / (float)cols;
    const T *dy = static_cast<const T *>(a.dy.data) + i * a.dy.group;
    const T *x = SAVED ? nullptr : static_cast<const T *>(a.x.data) + i * a.x.group;
    const uint8_t *codes = SAVED ? static_cast<const uint8_t *>(a.codes.data) + i * a.codes.group : nullptr;
    const float *scales = SAVED ? static_cast<const float *>(a.scales.data) + i * a.scales.group : nullptr;
    T *dx = DX ? static_cast<T *>(a.dx.data) + i * a.dx.group : nullptr;
    int at[kNV];
    bool mine[kNV];
    Two w[kNV][H], sw[kNV][H], sb[kNV][H];
#pragma unroll
    for (int v = 0; v < kNV; ++v) {
        at[v] = ((DX ? 0 : (int)blockIdx.z * kNV * TPR) + v * TPR + t) * N;       // without dx the columns may be cut
        mine[v] = at[v] < cols;
#pragma unroll
        for (int k = 0; k < H; ++k) {
            const P *from = static_cast<const P *>(a.w) + i * a.ldw + at[v] + 2 * k;
            w[v][k] = DX && mine[v] ? Two{value_of(from), value_of(from + 1)} : both(0.f);
            sw[v][k] = sb[v][k] = both(0.f);
        }
    }
    auto slot = [&](int stage, int v) { return (stage * kNV + v) * kThreadsHere + tid; };
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring), ring_x_at = (uint32_t)__cvta_generic_to_shared(ring_x),
                   ring_s_at = (uint32_t)__cvta_generic_to_shared(ring_s);
    auto fetch = [&](int stage, int64_t row) {
        if (row < last)
#pragma unroll
            for (int v = 0; v < kNV; ++v)
                if (mine[v]) {
                    cp_async<16>(ring_at + slot(stage, v) * 16, dy + row * a.dy.row + at[v]);
                    if (SAVED) {
                        cp_async<kXBytes>(ring_x_at + slot(stage, v) * kXBytes, codes + row * a.codes.row + at[v]);
                        cp_async<4>(ring_s_at + slot(stage, v) * 4, scales + row * a.scales.row + at[v] / ZENO_SAVED_BLOCK);
                    } else {
                        cp_async<16>(ring_x_at + slot(stage, v) * 16, x + row * a.x.row + at[v]);
                    }
                }
        cp_async_commit();
    };
#pragma unroll
    for (int q = 0; q < STAGES - 1; ++q) fetch(q, first + q * ROWS);
    int stage = 0, turn = 0;
    float mean = 0.f, rstd = 0.f;
    if (first < last) {
        mean = a.mean[i * a.n + first];
        rstd = a.rstd[i * a.n + first];
    }
    for (int64_t row = first; row - sub < last; row += ROWS) {
        float next_mean = 0.f, next_rstd = 0.f;
        if (row + ROWS < last) {
            next_mean = a.mean[i * a.n + row + ROWS];
            next_rstd = a.rstd[i * a.n + row + ROWS];
        }
        fetch(stage == 0 ? STAGES - 1 : stage - 1, row + (STAGES - 1) * ROWS);
        cp_async_wait<STAGES - 1>();
        const bool on = row < last;
        Two h[kNV][H], g[kNV][H], c1 = both(0.f), c2 = both(0.f);
#pragma unroll
        for (int v = 0; v < kNV; ++v) {
            Two d[H];
            pairs(reinterpret_cast<const uint4 *>(ring)[slot(stage, v)], d, T());
            if constexpr (SAVED) {
                const float scale = ring_s[slot(stage, v)];
                const uint32_t *c = reinterpret_cast<const uint32_t *>(ring_x + slot(stage, v) * kXBytes);
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    const __half2_raw e = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(c[k / 2] >> (16 * (k & 1))), __NV_E4M3);
                    const float2 f = __half22float2(__half2(e));
                    h[v][k] = mul2(Two{f.x, f.y}, both(scale));
                }
            } else {
                pairs(reinterpret_cast<const uint4 *>(ring_x)[slot(stage, v)], h[v], T());
            }
            // Where nothing was copied, the entry is the mean: (0 - mean) rstd of finite numbers may be beyond binary32, and its product with 0 a NaN.
            if (!on || !mine[v])
#pragma unroll
                for (int k = 0; k < H; ++k) d[k] = both(0.f), h[v][k] = both(mean);
#pragma unroll
            for (int k = 0; k < H; ++k) {
                h[v][k] = mul2(add2(h[v][k], both(-mean)), both(rstd));
                sw[v][k] = fma2(d[k], h[v][k], sw[v][k]);
                sb[v][k] = add2(sb[v][k], d[k]);
                g[v][k] = mul2(d[k], w[v][k]);
                c1 = add2(c1, g[v][k]);
                c2 = fma2(g[v][k], h[v][k], c2);
            }
        }
        if (DX) {
            Two c = {warp_sum(c1.x + c1.y), warp_sum(c2.x + c2.y)};
            if constexpr (kWarps > 1) {
                if ((t & 31) == 0) scratch[turn][sub][t >> 5] = make_float2(c.x, c.y);
                __syncthreads();
                const float4 *s = reinterpret_cast<const float4 *>(scratch[turn][sub]);
                c = both(0.f);
#pragma unroll
                for (int k = 0; k < kWarps / 2; ++k) {
                    const float4 v = s[k];
                    c = add2(c, add2(Two{v.x, v.y}, Two{v.z, v.w}));
                }
                turn ^= 1;
            }
            // rstd (g - c1 - h c2)
            const Two m1 = both(-rstd * c.x * inv), m2 = both(-rstd * c.y * inv), rs = both(rstd);
#pragma unroll
            for (int v = 0; v < kNV; ++v)
                if (on && mine[v]) {
                    Two o[H];
#pragma unroll
                    for (int k = 0; k < H; ++k) o[k] = fma2(h[v][k], m2, fma2(g[v][k], rs, m1));
                    *reinterpret_cast<uint4 *>(dx + row * a.dx.row + at[v]) = from_pairs(o, T());
                }
        }
        mean = next_mean;
        rstd = next_rstd;
        if (++stage == STAGES) stage = 0;
    }
    if (!a.dw && !a.db) return;
    cp_async_wait<0>();
    if constexpr (ROWS > 1) {
        float *joined = reinterpret_cast<float *>(ring);          // [ROWS - 1][2][NV][N][TPR]
        auto place = [&](int q, int which, int v, int k) { return joined + ((((q * 2 + which) * kNV + v) * N + k) * TPR) + t; };
        __syncthreads();
        if (sub > 0)
#pragma unroll
            for (int v = 0; v < kNV; ++v)
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    *place(sub - 1, 0, v, 2 * k) = sw[v][k].x;
                    *place(sub - 1, 0, v, 2 * k + 1) = sw[v][k].y;
                    *place(sub - 1, 1, v, 2 * k) = sb[v][k].x;
                    *place(sub - 1, 1, v, 2 * k + 1) = sb[v][k].y;
                }
        __syncthreads();
        if (sub > 0) return;
        for (int q = 0; q < ROWS - 1; ++q)
#pragma unroll
            for (int v = 0; v < kNV; ++v)
#pragma unroll
                for (int k = 0; k < H; ++k) {
                    sw[v][k].x += *place(q, 0, v, 2 * k);
                    sw[v][k].y += *place(q, 0, v, 2 * k + 1);
                    sb[v][k].x += *place(q, 1, v, 2 * k);
                    sb[v][k].y += *place(q, 1, v, 2 * k + 1);
                }
    }
#pragma unroll
    for (int v = 0; v < kNV; ++v) {
        if (!mine[v]) continue;
        if (part) {
            float *to = part + ((int64_t)i * chunks + blockIdx.x) * 2 * cols + at[v];       // cols is a multiple of N
#pragma unroll
            for (int k = 0; k < H; k += 2) {
                *reinterpret_cast<float4 *>(to + 2 * k) = make_float4(sw[v][k].x, sw[v][k].y, sw[v][k + 1].x, sw[v][k + 1].y);
                *reinterpret_cast<float4 *>(to + cols + 2 * k) = make_float4(sb[v][k].x, sb[v][k].y, sb[v][k + 1].x, sb[v][k + 1].y);
            }
            continue;
        }
#pragma unroll
        for (int k = 0; k < H; ++k) {
            const int64_t to = i * a.ldg + at[v] + 2 * k;
            if (a.dw) {
                put(static_cast<P *>(a.dw) + to, sw[v][k].x);
                put(static_cast<P *>(a.dw) + to + 1, sw[v][k].y);
            }
            if (a.db) {
                put(static_cast<P *>(a.db) + to, sb[v][k].x);
                put(static_cast<P *>(a.db) + to + 1, sb[v][k].y);
            }
        }
    }
}

// Rows of any alignment, and what is too long for the above: the columns blockIdx.x * TPR * NV .. of chunk blockIdx.z of a group's rows, R rows at
// a time with the next R on their way, one barrier for them all (7 x 333 x 777 binary32 from 8 bits: 13 us, a row at a time 26).  With DX the block has
// the whole row (gridDim.x is 1).
template <typename T, typename P, int TPR, int NV, int R, bool SAVED, bool DX>
__global__ void __launch_bounds__(TPR) norm_entries_kernel(NormGradArgs a, float *part) {
    constexpr int kWarps = TPR / 32;
    __shared__ float scratch[2][kWarps][2 * R];
    const int t = threadIdx.x, lane = t & 31, cols = (int)a.cols, chunks = gridDim.z, i = blockIdx.y;
    const int j0 = blockIdx.x * TPR * NV + t;
    const int64_t first = a.n * blockIdx.z / chunks, last = a.n * (blockIdx.z + 1) / chunks;
    const float inv = 1.f / (float)cols;
    const T *dy = static_cast<const T *>(a.dy.data) + i * a.dy.group + j0;
    const T *x = SAVED ? nullptr : static_cast<const T *>(a.x.data) + i * a.x.group + j0;
    const uint8_t *codes = SAVED ? static_cast<const uint8_t *>(a.codes.data) + i * a.codes.group + j0 : nullptr;
    const float *scales = SAVED ? static_cast<const float *>(a.scales.data) + i * a.scales.group : nullptr;
    float w[NV], sw[NV], sb[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        w[v] = DX && j0 + v * TPR < cols ? value_of(static_cast<const P *>(a.w) + i * a.ldw + j0 + v * TPR) : 0.f;
        sw[v] = sb[v] = 0.f;
    }
    // the next rows as they lie in memory: what is done to them waits until their turn
    T next_d[R][NV], next_x[SAVED ? 1 : R][SAVED ? 1 : NV];
    uint8_t next_c[SAVED ? R : 1][SAVED ? NV : 1];
    float next_s[SAVED ? R : 1][SAVED ? NV : 1], next_mean[R], next_rstd[R];
    auto fetch = [&](int64_t row0) {
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const int64_t row = row0 + q;
            if (row >= last) return;
            next_mean[q] = a.mean[i * a.n + row];
            next_rstd[q] = a.rstd[i * a.n + row];
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (j0 + v * TPR < cols) {
                    next_d[q][v] = dy[row * a.dy.row + v * TPR];
                    if constexpr (SAVED) {
                        next_c[q][v] = codes[row * a.codes.row + v * TPR];
                        next_s[q][v] = scales[row * a.scales.row + (j0 + v * TPR) / ZENO_SAVED_BLOCK];
                    } else {
                        next_x[q][v] = x[row * a.x.row + v * TPR];
                    }
                }
        }
    };
    fetch(first);
    int turn = 0;
    for (int64_t row = first; row < last; row += R) {
        float g[R][NV], h[R][NV], rs[R], c[2 * R];
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const bool on = row + q < last;
            rs[q] = on ? next_rstd[q] : 0.f;
            c[2 * q] = c[2 * q + 1] = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float d = 0.f;
                h[q][v] = 0.f;
                if (on && j0 + v * TPR < cols) {
                    d = value_of(&next_d[q][v]);
                    if constexpr (SAVED) h[q][v] = saved_value(next_c[q][v], next_s[q][v]);
                    else h[q][v] = value_of(&next_x[q][v]);
                    h[q][v] = (h[q][v] - next_mean[q]) * rs[q];
                }
                sw[v] = fmaf(d, h[q][v], sw[v]);
                sb[v] += d;
                g[q][v] = d * w[v];
                c[2 * q] += g[q][v];
                c[2 * q + 1] = fmaf(g[q][v], h[q][v], c[2 * q + 1]);
            }
        }
        fetch(row + R);
        if (!DX) continue;
        // the rows' sums, two for each: first a lane has one of them for the warp, then, over the warps, for the block
        float mine = warp_transpose_reduce<2 * R>(c, lane);
        if (lane < 2 * R) scratch[turn][t >> 5][lane] = mine;
        __syncthreads();
        mine = 0.f;
        constexpr int kGroups = 32 / (2 * R);
#pragma unroll
        for (int k = 0; k < kWarps; k += kGroups)
            if (k + lane / (2 * R) < kWarps) mine += scratch[turn][k + lane / (2 * R)][lane % (2 * R)];
#pragma unroll
        for (int k = 2 * R; k < 32; k <<= 1) mine += __shfl_xor_sync(0xffffffffu, mine, k);
        turn ^= 1;
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const float c1 = __shfl_sync(0xffffffffu, mine, 2 * q) * inv, c2 = __shfl_sync(0xffffffffu, mine, 2 * q + 1) * inv;
            if (row + q >= last) continue;
            T *dx = static_cast<T *>(a.dx.data) + i * a.dx.group + (row + q) * a.dx.row + j0;
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (j0 + v * TPR < cols) put(dx + v * TPR, rs[q] * (g[q][v] - c1 - h[q][v] * c2));
        }
    }
    if (!a.dw && !a.db) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int j = j0 + v * TPR;
        if (j >= cols) continue;
        if (part) {
            float *to = part + ((int64_t)i * chunks + blockIdx.z) * 2 * cols + j;
            to[0] = sw[v];
            to[cols] = sb[v];
        } else {
            if (a.dw) put(static_cast<P *>(a.dw) + i * a.ldg + j, sw[v]);
            if (a.db) put(static_cast<P *>(a.db) + i * a.ldg + j, sb[v]);
        }
    }
}

// Forward, many rows of up to 1024 vectors: TPR threads take R rows at a time, NV vectors of each in a thread's registers, with a group's
// weights in shared memory for all rows of the block.  (Taken from L2 for every row, as norm_row_kernel does, they cost as much of its
// bandwidth as the rows.)  Up to a warp's threads a row meets no barrier; two or four warps have one of their own.  A vector's
// register takes the next rows' vector as soon as its result is stored.  (21 x 2048 x 4096 bfloat16: 121 us, 5.8 TB/s.)
constexpr int kGroupThreads = 256;
template <typename T, typename P, int TPR, int NV, int R>
__global__ void __launch_bounds__(kGroupThreads, 2) norm_group_kernel(NormArgs a) {
    constexpr int N = 16 / sizeof(T), H = N / 2, kSide = kGroupThreads / TPR;        // rows side by side
    extern __shared__ __align__(16) float weights_at[];        // w, then b
    __shared__ float scratch[2][kGroupThreads / 32][R];
    const int t = threadIdx.x % TPR, side = threadIdx.x / TPR, cols = (int)a.cols, packs = cols / N, chunks = gridDim.x, i = blockIdx.y;
    const int64_t last = a.n * (blockIdx.x + 1) / chunks;
    int64_t row = a.n * blockIdx.x / chunks + side * R;
    const T *x = static_cast<const T *>(a.x.data) + i * a.x.group;
    T *y = static_cast<T *>(a.y.data) + i * a.y.group;
    uint4 raw[R][NV];
    auto fetch = [&](int q, int v, int64_t r) {
        const int at = v * TPR + t;
        raw[q][v] = make_uint4(0u, 0u, 0u, 0u);
        if (r < last && at < packs) raw[q][v] = reinterpret_cast<const uint4 *>(x + r * a.x.row)[at];
    };
#pragma unroll
    for (int q = 0; q < R; ++q)
#pragma unroll
        for (int v = 0; v < NV; ++v) fetch(q, v, row + q);
    // four weights of a thread beside the next one's, so that a warp's loads of 16 bytes meet all banks
    float *biases_at = weights_at + NV * TPR * N;
    for (int j = threadIdx.x; j < cols; j += kGroupThreads) {
        const int at = j / N, to = ((at / TPR * (N / 4) + j % N / 4) * TPR + at % TPR) * 4 + j % 4;
        weights_at[to] = value_of(static_cast<const P *>(a.w) + i * a.ldw + j);
        biases_at[to] = a.b ? value_of(static_cast<const P *>(a.b) + i * a.ldw + j) : 0.f;
    }
    __syncthreads();
    // the rows' averages in all of their threads
    auto averages = [&](float (&s)[R], int which) {
#pragma unroll
        for (int q = 0; q < R; ++q)
#pragma unroll
            for (int d = (TPR < 32 ? TPR : 32) / 2; d >= 1; d >>= 1) s[q] += __shfl_xor_sync(0xffffffffu, s[q], d);
        if constexpr (TPR > 32) {
            const int warp = threadIdx.x >> 5;
            if ((t & 31) == 0)
#pragma unroll
                for (int q = 0; q < R; ++q) scratch[which][warp][q] = s[q];
            asm volatile("bar.sync %0, %1;" ::"r"(side + 1), "n"(TPR) : "memory");
#pragma unroll
            for (int q = 0; q < R; ++q) {
                s[q] = 0.f;
#pragma unroll
                for (int k = 0; k < TPR / 32; ++k) s[q] += scratch[which][side * (TPR / 32) + k][q];
            }
        }
#pragma unroll
        for (int q = 0; q < R; ++q) s[q] /= (float)cols;
    };
    // a warp's threads go on together: up to where the first of their rows ends
    for (const int64_t behind = TPR < 32 ? (side % (32 / TPR)) * R : 0; row - behind < last; row += kSide * R) {
        float mean[R], rstd[R];
#pragma unroll
        for (int q = 0; q < R; ++q) {
            Two s = both(0.f);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                Two f[H];
                pairs(raw[q][v], f, T());
#pragma unroll
                for (int k = 0; k < H; ++k) s = add2(s, f[k]);
            }
            mean[q] = s.x + s.y;
        }
        averages(mean, 0);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            Two s = both(0.f);
#pragma unroll
            for (int v = 0; v < NV; ++v)
                if (v * TPR + t < packs) {
                    Two f[H];
                    pairs(raw[q][v], f, T());
#pragma unroll
                    for (int k = 0; k < H; ++k) {
                        f[k] = add2(f[k], both(-mean[q]));
                        s = fma2(f[k], f[k], s);
                    }
                }
            rstd[q] = s.x + s.y;
        }
        averages(rstd, 1);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            rstd[q] = rsqrtf(rstd[q] + a.eps);
            if (t == 0 && row + q < last) {
                if (a.mean) a.mean[i * a.n + row + q] = mean[q];
                if (a.rstd) a.rstd[i * a.n + row + q] = rstd[q];
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = v * TPR + t;
            Two w[H], b[H];
            if (at < packs)
#pragma unroll
                for (int k = 0; k < H; k += 2) {
                    const int from = ((v * (N / 4) + k / 2) * TPR + t) * 4;
                    const float4 wf = *reinterpret_cast<const float4 *>(weights_at + from), bf = *reinterpret_cast<const float4 *>(biases_at + from);
                    w[k] = Two{wf.x, wf.y};
                    w[k + 1] = Two{wf.z, wf.w};
                    b[k] = Two{bf.x, bf.y};
                    b[k + 1] = Two{bf.z, bf.w};
                }
#pragma unroll
            for (int q = 0; q < R; ++q) {
                if (at < packs && row + q < last) {
                    Two f[H];
                    pairs(raw[q][v], f, T());
#pragma unroll
                    for (int k = 0; k < H; ++k) f[k] = fma2(mul2(add2(f[k], both(-mean[q])), both(rstd[q])), w[k], b[k]);
                    reinterpret_cast<uint4 *>(y + (row + q) * a.y.row)[at] = from_pairs(f, T());
                }
                fetch(q, v, row + q + kSide * R);
            }
        }
    }
}

// The same for rows that start anywhere, by single entries: TPR threads take a row, NV of its entries in a thread's registers, the next row's on their
// way behind each result.  Every entry costs about a dozen instructions, four of them to memory of some kind.  (21 x 512 x 4096 in rows of 4097:
// bfloat16 57 us, binary32 78; by norm_row_kernel, where every row fetches its weights, 131 and 141.)
template <typename T, typename P, int TPR, int NV>
__global__ void __launch_bounds__(kGroupThreads, 4) norm_single_kernel(NormArgs a) {
    constexpr int kSide = kGroupThreads / TPR, kWarps = TPR / 32;
    extern __shared__ __align__(16) float weights_at[];        // w, then b
    __shared__ float scratch[2][kGroupThreads / 32];
    const int t = threadIdx.x % TPR, side = threadIdx.x / TPR, cols = (int)a.cols, chunks = gridDim.x, i = blockIdx.y;
    const int64_t last = a.n * (blockIdx.x + 1) / chunks;
    int64_t row = a.n * blockIdx.x / chunks + side;
    const T *x = static_cast<const T *>(a.x.data) + i * a.x.group + t;
    T *y = static_cast<T *>(a.y.data) + i * a.y.group + t;
    T raw[NV];
    auto fetch = [&](int v, int64_t r) {
        if (r < last && v * TPR + t < cols) raw[v] = x[r * a.x.row + v * TPR];
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) fetch(v, row);
    float *biases_at = weights_at + cols;
    for (int j = threadIdx.x; j < cols; j += kGroupThreads) {
        weights_at[j] = value_of(static_cast<const P *>(a.w) + i * a.ldw + j);
        biases_at[j] = a.b ? value_of(static_cast<const P *>(a.b) + i * a.ldw + j) : 0.f;
    }
    __syncthreads();
    // the row's average in all of its threads
    auto average = [&](float s, int which) {
        s = warp_sum(s);
        if constexpr (TPR > 32) {
            if ((t & 31) == 0) scratch[which][threadIdx.x >> 5] = s;
            asm volatile("bar.sync %0, %1;" ::"r"(side + 1), "n"(TPR) : "memory");
            s = 0.f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) s += scratch[which][side * kWarps + k];
        }
        return s / (float)cols;
    };
    for (; row < last; row += kSide) {
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (v * TPR + t < cols) s += value_of(raw + v);
        const float mean = average(s, 0);
        s = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
            if (v * TPR + t < cols) s = fmaf(value_of(raw + v) - mean, value_of(raw + v) - mean, s);
        const float rstd = rsqrtf(average(s, 1) + a.eps);
        if (t == 0) {
            if (a.mean) a.mean[i * a.n + row] = mean;
            if (a.rstd) a.rstd[i * a.n + row] = rstd;
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int j = v * TPR + t;
            if (j < cols) put(y + row * a.y.row + v * TPR, fmaf((value_of(raw + v) - mean) * rstd, weights_at[j], biases_at[j]));
            fetch(v, row + kSide);
        }
    }
}

// The blocks' sums of a group: 32 N columns a block, N a lane, eight warps take the blocks in turn.
template <typename P, int N>
__global__ void __launch_bounds__(kThreads) norm_join_kernel(const float *part, int chunks, int cols, P *dw, P *db, int64_t ldg) {
    constexpr int kWarps = kThreads / 32;
    __shared__ float sums[kWarps][N][32];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.y;
    const int64_t at = ((int64_t)blockIdx.x * 32 + lane) * N, all = 2 * (int64_t)cols;
    LongSum total[N];
    if (at < all)
        for (int c = warp; c < chunks;) {
            const int end = min(chunks, c + 2 * kShortSum * kWarps);          // one stretch for kNormBlocks of them
            float s[N];
#pragma unroll
            for (int k = 0; k < N; ++k) s[k] = 0.f;
#pragma unroll 4
            for (; c < end; c += kWarps) {
                const Pack<float, N> v = load_pack<float, N>(part + ((int64_t)i * chunks + c) * all + at);
#pragma unroll
                for (int k = 0; k < N; ++k) s[k] += v.v[k];
            }
#pragma unroll
            for (int k = 0; k < N; ++k) total[k].add(s[k]);
        }
#pragma unroll
    for (int k = 0; k < N; ++k) sums[warp][k][lane] = total[k].sum;
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * N; c += kThreads) {
        float v = 0.f;
#pragma unroll
        for (int q = 0; q < kWarps; ++q) v += sums[q][c % N][c / N];
        const int64_t to = (int64_t)blockIdx.x * 32 * N + c;
        P *out = to < cols ? dw : db;
        if (to < all && out) put(out + i * ldg + (to < cols ? to : to - cols), v);
    }
}

// Whether N weights (and biases) can be loaded at a time for every group.
template <typename P, int N>
bool wide_weights(const void *w, const void *b, int64_t ldw) {
    constexpr size_t kPack = N * sizeof(P) < 16 ? N * sizeof(P) : 16;
    return reinterpret_cast<uintptr_t>(w) % kPack == 0 && reinterpret_cast<uintptr_t>(b) % kPack == 0 && ldw * sizeof(P) % kPack == 0;
}

// Blocks that a group's rows are cut into: all groups' make two rounds of two blocks an SM, each block with at least 8 rows: few rows to a
// block are few groups' rows, whose sums stay in L2.  Long rows are cut into blocks by their columns too.
constexpr int kNormBlocks = 592;
int norm_chunks(int m, int64_t n, int64_t cols) {
    const int64_t by_columns = cols > 4096 ? cols / 4096 : 1;
    int64_t c = m > 0 ? kNormBlocks / (m * by_columns) : 1;
    if (c > n / 8) c = n / 8;
    return c < 1 ? 1 : (int)c;
}

// The same for the backward pass, with no more than 4,096 rows to a block (as far as a grid's third dimension goes): their sums are chains of additions.
constexpr int64_t kChainRows = 4096;
int gradient_chunks(int m, int64_t n, int64_t cols) {
    const int64_t c = min((n + kChainRows - 1) / kChainRows, (int64_t)65535);
    return (int)max((int64_t)norm_chunks(m, n, cols), c);
}

// sets a kernel's dynamic shared memory on the current device, once
template <typename K>
cudaError_t allow_shared(K *kernel, int bytes, PerDeviceOnce &once) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess && once.need(device)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess) once.mark(device);
    }
    return e;
}

template <typename T, typename P, int TPR, int NV, int R>
cudaError_t norm_groups(const NormArgs &a, cudaStream_t s) {
    constexpr int kSmem = 2 * NV * TPR * (16 / (int)sizeof(T)) * (int)sizeof(float);
    auto *kernel = norm_group_kernel<T, P, TPR, NV, R>;
    static PerDeviceOnce attr_set;
    const cudaError_t e = allow_shared(kernel, kSmem, attr_set);
    return e != cudaSuccess ? e : launch_chained(kernel, dim3(norm_chunks(a.m, a.n, 1), a.m), dim3(kGroupThreads), kSmem, s, false, a);
}

template <typename T, typename P, int TPR, int NV>
cudaError_t norm_singles(const NormArgs &a, cudaStream_t s) {
    static_assert(TPR * NV * 2 * (int)sizeof(float) <= 48 * 1024, "no attribute needed");
    return launch_chained(norm_single_kernel<T, P, TPR, NV>, dim3(norm_chunks(a.m, a.n, 1), a.m), dim3(kGroupThreads), 2 * (size_t)a.cols * sizeof(float), s, false, a);
}

template <typename T, typename P, int N, int TPR, int NV>
cudaError_t norm_rows(const NormArgs &a, bool wide, cudaStream_t s) {
    const int64_t rows = a.m * a.n;
    constexpr int kRows = TPR == 32 ? kRowBlock / 32 : 1;
    auto *kernel = N > 1 && wide ? norm_row_kernel<T, P, N, TPR, NV, true> : norm_row_kernel<T, P, N, TPR, NV, N == 1>;
    return launch_chained(kernel, dim3((unsigned)((rows + kRows - 1) / kRows)), dim3(TPR == 32 ? kRowBlock : TPR), 0, s, false, a, rows);
}

template <typename T, typename P>
cudaError_t layer_norm(const NormArgs &a, cudaStream_t s) {
    constexpr int N = 16 / sizeof(T);
    if (a.cols % N == 0 && aligned_to(a.x, a.m, a.n, sizeof(T), 16) && aligned_to(a.y, a.m, a.n, sizeof(T), 16)) {
        const bool wide = wide_weights<P, N>(a.w, a.b, a.ldw);
        const int64_t packs = a.cols / N;
        // Enough rows for two blocks an SM with eight rows each and more (21 x 2048 x 4096 bfloat16: 123 us, 157 by norm_row_kernel; 86,016 rows of
        // 128: 18 against 35).  Eight vectors a thread in bfloat16, whose weights take twice their bytes of shared memory; four in binary32
        // (43,008 rows of 4096: 227 us, with eight 258).
        if (norm_chunks(a.m, a.n, 1) * (int64_t)a.m >= kNormBlocks / 2 && a.n * a.m >= kNormBlocks * 8 && packs <= 1024) {
            constexpr int kMany = sizeof(T) == 2 ? 8 : 4;
            if (packs <= 16) return norm_groups<T, P, 4, 4, 2>(a, s);
            if (packs <= 32) return norm_groups<T, P, 8, 4, 2>(a, s);
            if (packs <= 64) return norm_groups<T, P, 16, 4, 2>(a, s);
            if (packs <= 128) return norm_groups<T, P, 32, 4, 2>(a, s);
            if (packs <= 256) return norm_groups<T, P, 256 / kMany, kMany, 1>(a, s);
            if (packs <= 512) return norm_groups<T, P, 512 / kMany, kMany, 1>(a, s);
            return norm_groups<T, P, 1024 / kMany, kMany, 1>(a, s);
        }
        if (packs <= 32) return norm_rows<T, P, N, 32, 1>(a, wide, s);
        if (packs <= 64) return norm_rows<T, P, N, 32, 2>(a, wide, s);
        if (packs <= 128) return norm_rows<T, P, N, 32, 4>(a, wide, s);
        if (packs <= 256) return norm_rows<T, P, N, 64, 4>(a, wide, s);
        if (packs <= 512) return norm_rows<T, P, N, 128, 4>(a, wide, s);
        if (packs <= 1024) return norm_rows<T, P, N, 256, 4>(a, wide, s);
        if (packs <= 2048) return norm_rows<T, P, N, 512, 4>(a, wide, s);
        if (packs <= 4096) return norm_rows<T, P, N, 1024, 4>(a, wide, s);
    } else {
        // A block an SM with eight rows each and more (1 x 1200 x 4095 bfloat16: 20 us, 22 by norm_row_kernel; 3 x 300 binary32: 26 and 22)
        if (norm_chunks(a.m, a.n, 1) * (int64_t)a.m >= kNormBlocks / 4 && a.n * a.m >= kNormBlocks * 2) {
            if (a.cols <= 256) return norm_singles<T, P, 32, 8>(a, s);
            if (a.cols <= 1024) return norm_singles<T, P, 64, 16>(a, s);
            if (a.cols <= 4096) return norm_singles<T, P, 256, 16>(a, s);
        }
        if (a.cols <= 256) return norm_rows<T, P, 1, 32, 8>(a, false, s);
        if (a.cols <= 1024) return norm_rows<T, P, 1, 64, 16>(a, false, s);
        if (a.cols <= 4096) return norm_rows<T, P, 1, 256, 16>(a, false, s);
        if (a.cols <= 16384) return norm_rows<T, P, 1, 1024, 16>(a, false, s);
    }
    return launch_chained(norm_any_kernel<T, P>, dim3((unsigned)(a.m * a.n)), dim3(kThreads), 0, s, false, a);
}

template <typename P>
cudaError_t norm_join(const NormGradArgs &a, int chunks, cudaStream_t s) {
    const int n = a.cols % 4 == 0 ? 4 : 1;
    return launch_chained(n == 4 ? norm_join_kernel<P, 4> : norm_join_kernel<P, 1>, dim3((unsigned)((2 * a.cols + 32 * n - 1) / (32 * n)), a.m), dim3(kThreads),
                          0, s, true, a.workspace, chunks, (int)a.cols, static_cast<P *>(a.dw), static_cast<P *>(a.db), a.ldg);
}

template <typename T, typename P, int TPR, bool SAVED, bool DX>
cudaError_t norm_columns(const NormGradArgs &a, cudaStream_t s) {
    constexpr int kRows = TPR < 256 ? 256 / TPR : 1, kStages = TPR <= 256 ? 4 : 3;
    constexpr int kSmem = kStages * kNV * TPR * kRows * (kSlotBytes<T, SAVED> + (SAVED ? 4 : 0));
    auto *kernel = norm_columns_kernel<T, P, TPR, kRows, kStages, SAVED, DX>;
    static PerDeviceOnce attr_set;
    cudaError_t e = allow_shared(kernel, kSmem, attr_set);
    if (e != cudaSuccess) return e;
    const int chunks = gradient_chunks(a.m, a.n, a.cols);
    const bool join = (a.dw || a.db) && chunks > 1;
    const int64_t per_block = (int64_t)TPR * kNV * (16 / sizeof(T)), tiles = DX ? 1 : (a.cols + per_block - 1) / per_block;
    e = launch_chained(kernel, dim3(chunks, a.m, (unsigned)tiles), dim3(TPR * kRows), kSmem, s, false, a, join ? a.workspace : nullptr);
    return e == cudaSuccess && join ? norm_join<P>(a, chunks, s) : e;
}

template <typename T, typename P, bool SAVED, bool DX>
cudaError_t norm_columns_any(const NormGradArgs &a, cudaStream_t s) {
    const int64_t packs = a.cols / (16 / sizeof(T));
    if (packs <= 64) return norm_columns<T, P, 32, SAVED, DX>(a, s);
    if (packs <= 128) return norm_columns<T, P, 64, SAVED, DX>(a, s);
    if (packs <= 256) return norm_columns<T, P, 128, SAVED, DX>(a, s);
    if (packs <= 512) return norm_columns<T, P, 256, SAVED, DX>(a, s);
    return norm_columns<T, P, 512, SAVED, DX>(a, s);
}

template <typename T, typename P, int TPR, int NV, int R, bool DX>
cudaError_t norm_entries(const NormGradArgs &a, cudaStream_t s) {
    const int64_t tiles = DX ? 1 : (a.cols + TPR * NV - 1) / (TPR * NV);
    const int chunks = gradient_chunks(a.m, a.n, a.cols);
    const bool join = (a.dw || a.db) && chunks > 1;
    auto *kernel = a.x.data || a.n == 0 ? norm_entries_kernel<T, P, TPR, NV, R, false, DX> : norm_entries_kernel<T, P, TPR, NV, R, true, DX>;
    const cudaError_t e = launch_chained(kernel, dim3((unsigned)tiles, a.m, chunks), dim3(TPR), 0, s, false, a, join ? a.workspace : nullptr);
    return e == cudaSuccess && join ? norm_join<P>(a, chunks, s) : e;
}

template <typename T, typename P, int N, int TPR, int NV>
cudaError_t norm_dx_row(const NormGradArgs &a, cudaStream_t s) {
    const bool wide = N > 1 && wide_weights<P, N>(a.w, nullptr, a.ldw);
    auto *kernel = a.x.data ? (wide ? norm_dx_row_kernel<T, P, N, TPR, NV, false, (N > 1)> : norm_dx_row_kernel<T, P, N, TPR, NV, false, false>)
                            : (wide ? norm_dx_row_kernel<T, P, N, TPR, NV, true, (N > 1)> : norm_dx_row_kernel<T, P, N, TPR, NV, true, false>);
    return launch_chained(kernel, dim3((unsigned)(a.m * a.n)), dim3(TPR), 0, s, false, a);
}

template <typename T, typename P>
cudaError_t layer_norm_gradient(const NormGradArgs &a, cudaStream_t s) {
    constexpr int N = 16 / sizeof(T);
    const bool dx = a.dx.data && a.n > 0, weights = a.dw || a.db;
    const bool aligned = a.cols % N == 0 && aligned_to(a.dy, a.m, a.n, sizeof(T), 16) && aligned_to(a.dx, a.m, a.n, sizeof(T), 16) &&
                         (a.x.data ? aligned_to(a.x, a.m, a.n, sizeof(T), 16) : aligned_to(a.codes, a.m, a.n, 1, N));
    if (!dx && !weights) return cudaSuccess;
    if (a.n > 0 && aligned && a.cols <= 1024 * N) {
        if (a.x.data) return dx ? norm_columns_any<T, P, false, true>(a, s) : norm_columns_any<T, P, false, false>(a, s);
        return dx ? norm_columns_any<T, P, true, true>(a, s) : norm_columns_any<T, P, true, false>(a, s);
    }
    if (dx && weights) {
        if (a.cols <= 256) return norm_entries<T, P, 64, 4, 4, true>(a, s);
        if (a.cols <= 512) return norm_entries<T, P, 128, 4, 4, true>(a, s);
        if (a.cols <= 1024) return norm_entries<T, P, 256, 4, 4, true>(a, s);
        if (a.cols <= 2048) return norm_entries<T, P, 512, 4, 2, true>(a, s);
        if (a.cols <= 4096) return norm_entries<T, P, 1024, 4, 1, true>(a, s);
    }
    // long rows: the weight gradients, then dx, each from a reading of its own; dx last, since it may lie in dy's place
    cudaError_t e = cudaSuccess;
    if (weights) {
        if (a.n > 0 && aligned) e = a.x.data ? norm_columns<T, P, 256, false, false>(a, s) : norm_columns<T, P, 256, true, false>(a, s);
        else e = norm_entries<T, P, 256, 2, 4, false>(a, s);
    }
    if (e != cudaSuccess || !dx) return e;
    if (aligned && a.cols <= 2048 * N) return norm_dx_row<T, P, N, 512, 4>(a, s);
    if (aligned && a.cols <= 4096 * N) return norm_dx_row<T, P, N, 1024, 4>(a, s);
    if (a.cols <= 8192) return norm_dx_row<T, P, 1, 1024, 8>(a, s);
    if (a.cols <= 16384) return norm_dx_row<T, P, 1, 1024, 16>(a, s);
    return launch_chained(norm_dx_any_kernel<T, P>, dim3((unsigned)(a.m * a.n)), dim3(kThreads), 0, s, false, a);
}

}  // namespace

cudaError_t launch_layer_norm(int type, int param_type, const NormArgs &a, cudaStream_t s) {
    if (type == ZENO_BF16)
        return param_type == ZENO_BF16 ? layer_norm<__nv_bfloat16, __nv_bfloat16>(a, s) : layer_norm<__nv_bfloat16, float>(a, s);
    return param_type == ZENO_BF16 ? layer_norm<float, __nv_bfloat16>(a, s) : layer_norm<float, float>(a, s);
}

int64_t norm_gradient_workspace(int m, int64_t n, int64_t cols) {
    const int chunks = gradient_chunks(m, n, cols);
    return chunks > 1 ? (int64_t)m * chunks * 2 * cols * (int64_t)sizeof(float) : 0;
}

cudaError_t launch_layer_norm_gradient(int type, int param_type, const NormGradArgs &a, cudaStream_t s) {
    if (type == ZENO_BF16)
        return param_type == ZENO_BF16 ? layer_norm_gradient<__nv_bfloat16, __nv_bfloat16>(a, s) : layer_norm_gradient<__nv_bfloat16, float>(a, s);
    return param_type == ZENO_BF16 ? layer_norm_gradient<float, __nv_bfloat16>(a, s) : layer_norm_gradient<float, float>(a, s);
}

}  // namespace zeno

// Layer norm of rows of activations, and its backward pass with the weight gradients reduced per group (worker).
//
// Bound by the activations' bytes: forward x in, y out; backward dy and x in, dx out, each once.  Forward: a row's entries stay in
// the registers of the 32 to 1024 threads that share it, between the sum, the centred squares and the result.  Backward: a
// thread owns columns, not rows: it goes down a stretch of a group's rows with the sums of its columns' weight gradients in
// registers, and the loads of the rows ahead are in flight while a row's two averages are formed across the block.
#include "zeno_operators.h"
#include "zeno_saved.cuh"

namespace zeno {

namespace {

constexpr int kThreads = 256;

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
    float s = 0.f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) s += value_of(x + j);
    const float mean = block_sum<kThreads>(s, scratch[0]) / (float)a.cols;
    s = 0.f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
        const float d = value_of(x + j) - mean;
        s = fmaf(d, d, s);
    }
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
    float s1 = 0.f, s2 = 0.f;
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
        const float g = value_of(dy + j) * value_of(w + j);
        s1 += g;
        s2 = fmaf(g, (x(j) - mean) * rstd, s2);
    }
    const float c1 = block_sum<kThreads>(s1, scratch[0]) / (float)a.cols, c2 = block_sum<kThreads>(s2, scratch[1]) / (float)a.cols;
    for (int64_t j = threadIdx.x; j < a.cols; j += kThreads) {
        const float g = value_of(dy + j) * value_of(w + j), h = (x(j) - mean) * rstd;
        put(dx + j, rstd * (g - c1 - h * c2));
    }
}

// Weight gradients: a block takes 32 columns of a group, its warps the group's rows in turn.
template <typename T, typename P>
__global__ void __launch_bounds__(kThreads) norm_weights_any_kernel(NormGradArgs a) {
    constexpr int kWarps = kThreads / 32;
    __shared__ float sums[2][kWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t j = (int64_t)blockIdx.x * 32 + lane;
    const int i = blockIdx.y;
    float sw = 0.f, sb = 0.f;
    if (j < a.cols)
        for (int64_t t = warp; t < a.n; t += kWarps) {
            const int64_t r = i * a.n + t;
            const float d = value_of(static_cast<const T *>(a.dy.data) + a.dy.at(r) + j);
            sw = fmaf(d, (InputRow<T>(a, r)(j) - a.mean[r]) * a.rstd[r], sw);
            sb += d;
        }
    sums[0][warp][lane] = sw;
    sums[1][warp][lane] = sb;
    __syncthreads();
    if (warp < 2 && j < a.cols) {
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < kWarps; ++q) s += sums[warp][q][lane];
        void *out = warp == 0 ? a.dw : a.db;
        if (out) put(static_cast<P *>(out) + i * a.ldg + j, s);
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

// A row in TPR threads, NV packs of N entries each.  WV: the weights can be loaded N at a time too.
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

// ---- backward, by columns

// The layer's input, N entries at a time: as it was, or codes and their block's scale
template <typename T, int N, bool SAVED> struct InputPack;
template <typename T, int N> struct InputPack<T, N, false> {
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

// A block: ROWS rows side by side, TPR threads each, N columns a thread, down the rows [first, last) of group blockIdx.y.  Then
// the sums of the ROWS rows' threads are joined, and go to the group's gradients, or (several blocks to a group) to `part`
// [group][block][dw, db][cols].
template <typename T, typename P, int N, int TPR, int ROWS, bool SAVED, bool DX>
__global__ void __launch_bounds__(TPR *ROWS) norm_columns_kernel(NormGradArgs a, float *part) {
    constexpr int kWarps = TPR / 32;
    constexpr int kAhead = TPR * N >= 8192 ? 1 : 2;      // rows whose loads are in flight ahead of the one at work: 64 registers a thread
    __shared__ float2 scratch[2][kWarps];
    __shared__ float joined[ROWS > 1 ? 2 : 1][ROWS > 1 ? (ROWS - 1) * TPR * N : 1];
    const int sub = ROWS > 1 ? threadIdx.x / TPR : 0, t = ROWS > 1 ? threadIdx.x % TPR : threadIdx.x;
    const int cols = (int)a.cols, j = t * N, chunks = gridDim.x, i = blockIdx.y;
    const bool mine = j < cols;
    const int64_t first = a.n * blockIdx.x / chunks, last = a.n * (blockIdx.x + 1) / chunks;
    const float inv = 1.f / (float)cols;
    float w[N], sw[N], sb[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        w[k] = DX && mine ? value_of(static_cast<const P *>(a.w) + i * a.ldw + j + k) : 0.f;
        sw[k] = sb[k] = 0.f;
    }
    Pack<T, N> dy[kAhead];
    InputPack<T, N, SAVED> x[kAhead];
    float mean[kAhead], rstd[kAhead];
    auto fetch = [&](int slot, int64_t row) {
        if (row >= last) return;
        const int64_t r = i * a.n + row;
        mean[slot] = a.mean[r];
        rstd[slot] = a.rstd[r];
        if (!mine) return;
        dy[slot] = load_pack<T, N>(static_cast<const T *>(a.dy.data) + a.dy.at(r) + j);
        x[slot].load(a, r, j);
    };
#pragma unroll
    for (int q = 0; q < kAhead; ++q) fetch(q, first + sub + q * ROWS);
    int turn = 0;
    for (int64_t row0 = first; row0 < last; row0 += kAhead * ROWS)
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int64_t row = row0 + q * ROWS + sub;
            if (row0 + q * ROWS >= last) break;           // the whole block's
            const bool on = row < last && mine;
            float g[N], h[N], d[N], c1 = 0.f, c2 = 0.f;
            const float rs = row < last ? rstd[q] : 0.f, mu = row < last ? mean[q] : 0.f;
            if (on) {
                values(dy[q], d);
                x[q].get(h);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    h[k] = (h[k] - mu) * rs;
                    sw[k] = fmaf(d[k], h[k], sw[k]);
                    sb[k] += d[k];
                    g[k] = d[k] * w[k];
                    c1 += g[k];
                    c2 = fmaf(g[k], h[k], c2);
                }
            }
            fetch(q, row + kAhead * ROWS);
            if (!DX) continue;
            c1 = warp_sum(c1);
            c2 = warp_sum(c2);
            if constexpr (kWarps > 1) {                   // ROWS is 1 then
                if ((t & 31) == 0) scratch[turn][t >> 5] = make_float2(c1, c2);
                __syncthreads();
                c1 = c2 = 0.f;
#pragma unroll
                for (int k = 0; k < kWarps; ++k) {
                    const float2 v = scratch[turn][k];
                    c1 += v.x;
                    c2 += v.y;
                }
                turn ^= 1;
            }
            if (on) {
                c1 *= inv;
                c2 *= inv;
#pragma unroll
                for (int k = 0; k < N; ++k) g[k] = rs * (g[k] - c1 - h[k] * c2);
                store_pack<T, N>(static_cast<T *>(a.dx.data) + a.dx.at(i * a.n + row) + j, g);
            }
        }
    if (!a.dw && !a.db) return;
    if constexpr (ROWS > 1) {
        if (sub > 0)
#pragma unroll
            for (int k = 0; k < N; ++k) {
                joined[0][((sub - 1) * TPR + t) * N + k] = sw[k];
                joined[1][((sub - 1) * TPR + t) * N + k] = sb[k];
            }
        __syncthreads();
        if (sub > 0) return;
        for (int q = 0; q < ROWS - 1; ++q)
#pragma unroll
            for (int k = 0; k < N; ++k) {
                sw[k] += joined[0][(q * TPR + t) * N + k];
                sb[k] += joined[1][(q * TPR + t) * N + k];
            }
    }
    if (!mine) return;
    if (part) {
        float *to = part + ((int64_t)i * chunks + blockIdx.x) * 2 * cols + j;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            to[k] = sw[k];
            to[cols + k] = sb[k];
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (a.dw) put(static_cast<P *>(a.dw) + i * a.ldg + j + k, sw[k]);
        if (a.db) put(static_cast<P *>(a.db) + i * a.ldg + j + k, sb[k]);
    }
}

// The blocks' sums of a group, column by column: 32 columns a block, eight warps take the blocks in turn.
template <typename P>
__global__ void __launch_bounds__(kThreads) norm_join_kernel(const float *part, int chunks, int cols, P *dw, P *db, int64_t ldg) {
    constexpr int kWarps = kThreads / 32;
    __shared__ float sums[kWarps][32];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.y;
    const int at = blockIdx.x * 32 + lane;           // of the 2 cols sums
    float s = 0.f;
    if (at < 2 * cols)
#pragma unroll 4
        for (int c = warp; c < chunks; c += kWarps) s += part[((int64_t)i * chunks + c) * 2 * cols + at];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && at < 2 * cols) {
#pragma unroll
        for (int q = 1; q < kWarps; ++q) s += sums[q][lane];
        P *out = at < cols ? dw : db;
        if (out) put(out + i * ldg + (at < cols ? at : at - cols), s);
    }
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
        const size_t pack = N * sizeof(P) < 16 ? N * sizeof(P) : 16;
        const bool wide = reinterpret_cast<uintptr_t>(a.w) % pack == 0 && reinterpret_cast<uintptr_t>(a.b) % pack == 0 && a.ldw * sizeof(P) % pack == 0;
        const int64_t packs = a.cols / N;
        if (packs <= 32) return norm_rows<T, P, N, 32, 1>(a, wide, s);
        if (packs <= 64) return norm_rows<T, P, N, 32, 2>(a, wide, s);
        if (packs <= 128) return norm_rows<T, P, N, 32, 4>(a, wide, s);
        if (packs <= 256) return norm_rows<T, P, N, 64, 4>(a, wide, s);
        if (packs <= 512) return norm_rows<T, P, N, 128, 4>(a, wide, s);
        if (packs <= 1024) return norm_rows<T, P, N, 256, 4>(a, wide, s);
        if (packs <= 2048) return norm_rows<T, P, N, 512, 4>(a, wide, s);
        if (packs <= 4096) return norm_rows<T, P, N, 1024, 4>(a, wide, s);
    } else {
        if (a.cols <= 256) return norm_rows<T, P, 1, 32, 8>(a, false, s);
        if (a.cols <= 1024) return norm_rows<T, P, 1, 64, 16>(a, false, s);
        if (a.cols <= 4096) return norm_rows<T, P, 1, 256, 16>(a, false, s);
        if (a.cols <= 16384) return norm_rows<T, P, 1, 1024, 16>(a, false, s);
    }
    return launch_chained(norm_any_kernel<T, P>, dim3((unsigned)(a.m * a.n)), dim3(kThreads), 0, s, false, a);
}

// Blocks that a group's rows are cut into.  About four times as many blocks as SMs (two at a time, so two rounds), each with at least
// 16 rows for every row of threads.
constexpr int kNormBlocks = 592;
int norm_chunks(int m, int64_t n) {
    int64_t c = m > 0 ? kNormBlocks / m : 1;
    if (c > n / 16) c = n / 16;
    return c < 1 ? 1 : (int)c;
}

template <typename T, typename P, int N, int TPR, int ROWS>
cudaError_t norm_columns(const NormGradArgs &a, cudaStream_t s) {
    const bool weights = a.dw || a.db, saved = !a.x.data;
    const int chunks = norm_chunks(a.m, a.n);
    auto *kernel = a.dx.data ? (saved ? norm_columns_kernel<T, P, N, TPR, ROWS, true, true> : norm_columns_kernel<T, P, N, TPR, ROWS, false, true>)
                             : (saved ? norm_columns_kernel<T, P, N, TPR, ROWS, true, false> : norm_columns_kernel<T, P, N, TPR, ROWS, false, false>);
    const bool join = weights && chunks > 1;
    cudaError_t e = launch_chained(kernel, dim3(chunks, a.m), dim3(TPR * ROWS), 0, s, false, a, join ? a.workspace : nullptr);
    if (e == cudaSuccess && join)
        e = launch_chained(norm_join_kernel<P>, dim3((unsigned)((2 * a.cols + 31) / 32), a.m), dim3(kThreads), 0, s, true, a.workspace, chunks,
                           (int)a.cols, static_cast<P *>(a.dw), static_cast<P *>(a.db), a.ldg);
    return e;
}

template <typename T, typename P, int N>
cudaError_t norm_columns_any(const NormGradArgs &a, cudaStream_t s) {
    const int64_t packs = a.cols / N;
    if (packs <= 32) return norm_columns<T, P, N, 32, 8>(a, s);
    if (packs <= 64) return norm_columns<T, P, N, 64, 1>(a, s);
    if (packs <= 128) return norm_columns<T, P, N, 128, 1>(a, s);
    if (packs <= 256) return norm_columns<T, P, N, 256, 1>(a, s);
    if (packs <= 512) return norm_columns<T, P, N, 512, 1>(a, s);
    return norm_columns<T, P, N, 1024, 1>(a, s);
}

template <typename T, typename P>
cudaError_t layer_norm_gradient(const NormGradArgs &a, cudaStream_t s) {
    constexpr int N = 16 / sizeof(T);
    const bool aligned = a.cols % N == 0 && aligned_to(a.dy, a.m, a.n, sizeof(T), 16) && aligned_to(a.dx, a.m, a.n, sizeof(T), 16) &&
                         (a.x.data ? aligned_to(a.x, a.m, a.n, sizeof(T), 16) : aligned_to(a.codes, a.m, a.n, 1, N));
    if (a.n > 0 && aligned && a.cols <= 1024 * N) return norm_columns_any<T, P, N>(a, s);
    if (a.n > 0 && a.cols <= 1024) return norm_columns_any<T, P, 1>(a, s);
    cudaError_t e = cudaSuccess;
    if (a.dw || a.db) e = launch_chained(norm_weights_any_kernel<T, P>, dim3((unsigned)((a.cols + 31) / 32), a.m), dim3(kThreads), 0, s, false, a);
    // last, since dx may lie in dy's place
    if (e == cudaSuccess && a.dx.data && a.n > 0)
        e = launch_chained(norm_dx_any_kernel<T, P>, dim3((unsigned)(a.m * a.n)), dim3(kThreads), 0, s, false, a);
    return e;
}

}  // namespace

cudaError_t launch_layer_norm(int type, int param_type, const NormArgs &a, cudaStream_t s) {
    if (type == ZENO_BF16)
        return param_type == ZENO_BF16 ? layer_norm<__nv_bfloat16, __nv_bfloat16>(a, s) : layer_norm<__nv_bfloat16, float>(a, s);
    return param_type == ZENO_BF16 ? layer_norm<float, __nv_bfloat16>(a, s) : layer_norm<float, float>(a, s);
}

int64_t norm_gradient_workspace(int m, int64_t n, int64_t cols) {
    const int chunks = norm_chunks(m, n);
    return chunks > 1 ? (int64_t)m * chunks * 2 * cols * (int64_t)sizeof(float) : 0;
}

cudaError_t launch_layer_norm_gradient(int type, int param_type, const NormGradArgs &a, cudaStream_t s) {
    if (type == ZENO_BF16)
        return param_type == ZENO_BF16 ? layer_norm_gradient<__nv_bfloat16, __nv_bfloat16>(a, s) : layer_norm_gradient<__nv_bfloat16, float>(a, s);
    return param_type == ZENO_BF16 ? layer_norm_gradient<float, __nv_bfloat16>(a, s) : layer_norm_gradient<float, float>(a, s);
}

}  // namespace zeno

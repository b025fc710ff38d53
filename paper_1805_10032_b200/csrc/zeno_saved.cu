// Activations kept in 8 bits for the backward pass, and the dense layers' weight gradients that are taken from them.
#include "zeno_saved.cuh"

namespace zeno {

namespace {

constexpr int kBlock = ZENO_SAVED_BLOCK;
constexpr int kMinExp = -117, kMaxExp = 119;

// bits of |v| if it is finite, else 0: non-finite entries do not count for a block's maximum
__device__ __forceinline__ uint32_t finite_bits(float v) {
    const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

// k of a block's scale 2^k: amax = f 2^e with 1 <= f < 2 is at most 448 2^k = 1.75 2^(k+8) from k = e - 8 on if f <= 1.75, else
// from e - 7 on.  Subnormal maxima are far below the smallest k.
__device__ __forceinline__ int scale_exponent(uint32_t amax) {
    const int k = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7fffffu) > 0x600000u);
    return min(max(k, kMinExp), kMaxExp);
}

// one code: to nearest even; the conversion saturates, and infinities are made NaN like NaN itself
__device__ __forceinline__ uint8_t code_of(float v, float inv_scale) {
    const float q = fabsf(v) < INFINITY ? v * inv_scale : NAN;
    return (uint8_t)__nv_cvt_float_to_fp8(q, __NV_SATFINITE, __NV_E4M3);
}

// Codes of any alignment: a warp takes a block of one row.
template <typename T>
__global__ void __launch_bounds__(256) pack_any_kernel(PackArgs a, int64_t blocks_per_row, int64_t blocks) {
    const int lane = threadIdx.x & 31;
    for (int64_t q = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); q < blocks; q += (int64_t)gridDim.x * 8) {
        const int64_t r = q / blocks_per_row, blk = q - r * blocks_per_row;
        const T *x = static_cast<const T *>(a.x.data) + a.x.at(r) + blk * kBlock;
        uint8_t *codes = static_cast<uint8_t *>(a.codes.data) + a.codes.at(r) + blk * kBlock;
        const int count = (int)min((int64_t)kBlock, a.cols - blk * kBlock);
        float v[kBlock / 32];
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < kBlock / 32; ++i) {
            v[i] = lane + 32 * i < count ? value_of(x + lane + 32 * i) : 0.f;
            amax = max(amax, finite_bits(v[i]));
        }
        amax = __reduce_max_sync(0xffffffffu, amax);
        const int k = amax ? scale_exponent(amax) : 0;
        const float inv = __uint_as_float((uint32_t)(127 - k) << 23);
#pragma unroll
        for (int i = 0; i < kBlock / 32; ++i)
            if (lane + 32 * i < count) codes[lane + 32 * i] = code_of(v[i], inv);
        if (lane == 0) (static_cast<float *>(a.scales.data) + a.scales.at(r))[blk] = __uint_as_float((uint32_t)(127 + k) << 23);
    }
}

// 16 lanes take a block, eight columns each; a half-warp takes kStrip blocks of a row one behind the
// other, with all their loads ahead of the first maximum.  The maxima of four blocks go over the lanes together, and one lane in four works a block's
// scale out: 9 shuffles instead of 16, a quarter of the scales' arithmetic.  Bound by bytes (20 x 2048 x 4096: bfloat16 84 us, 6.1 TB/s, 88 block by
// block; binary32 127 us, 6.7 TB/s).
//
// Rows that start anywhere (WHOLE false) are read by the aligned 16 bytes that a lane's entries lie in, one more than there would be, and put
// together by shifts, which are the same for all of a row; 20 x 512 x 4096 in rows of 4097: bfloat16 38 us,
// binary32 58, either 100 by single entries.
constexpr int kStrip = 4;

// Eight entries of a row: the bits of their largest magnitude (at least 0x7f800000 if one is not finite), and themselves as pairs.
struct Eight {
    uint4 u, v;
    __device__ __forceinline__ void load(const float *p) {
        u = __ldcs(reinterpret_cast<const uint4 *>(p));
        v = __ldcs(reinterpret_cast<const uint4 *>(p) + 1);
    }
    __device__ __forceinline__ uint32_t most(float) const {
        const uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7fffffffu);
        return m;
    }
    __device__ __forceinline__ void get(Two (&f)[4], float) const {
        f[0] = Two{__uint_as_float(u.x), __uint_as_float(u.y)};
        f[1] = Two{__uint_as_float(u.z), __uint_as_float(u.w)};
        f[2] = Two{__uint_as_float(v.x), __uint_as_float(v.y)};
        f[3] = Two{__uint_as_float(v.z), __uint_as_float(v.w)};
    }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { u = __ldcs(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ uint32_t most(__nv_bfloat16) const {
        auto size = [](uint32_t w) {
            w &= 0x7fff7fffu;
            return *reinterpret_cast<__nv_bfloat162 *>(&w);
        };
        const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(size(u.x), size(u.y)), __hmax2_nan(size(u.z), size(u.w)));
        const uint32_t w = *reinterpret_cast<const uint32_t *>(&m);
        return max(w << 16, w & 0xffff0000u);
    }
    __device__ __forceinline__ void get(Two (&f)[4], __nv_bfloat16) const {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = Two{__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)};
    }
};

// Eight entries that start anywhere.  `from` and `to`: where the first and behind the last entry of the group's rows lie; what is in between may be
// read, whosever it is.
template <typename T> struct Shifted {
    static constexpr int kWords = 2 * sizeof(T);                  // of eight entries
    uint4 raw[kWords / 4 + 1];
    unsigned off;
    __device__ __forceinline__ void load(const T *p, int count, uintptr_t from, uintptr_t to) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p), first = at & ~(uintptr_t)15;
        off = (unsigned)(at & 15);
#pragma unroll
        for (int i = 0; i <= kWords / 4; ++i) raw[i] = make_uint4(0u, 0u, 0u, 0u);
        const uintptr_t end = at + count * sizeof(T);
        if (count > 0 && first >= from && ((end + 15) & ~(uintptr_t)15) <= to) {
#pragma unroll
            for (int i = 0; i <= kWords / 4; ++i)
                if (first + i * 16 < end) raw[i] = __ldcs(reinterpret_cast<const uint4 *>(first) + i);
        } else {                                                  // at the ends of the group's rows
            uint32_t w[kWords] = {};
            constexpr int kPer = 4 / sizeof(T);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) {
                    uint32_t bits;
                    if constexpr (kPer == 1) bits = reinterpret_cast<const uint32_t *>(p)[i];
                    else bits = reinterpret_cast<const uint16_t *>(p)[i];
                    w[i / kPer] |= bits << (i % kPer * 16);
                }
            off = 0;
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) raw[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
    }
    // the entries, those from `count` on zero
    __device__ __forceinline__ Eight get(int count) const {
        Eight e;
        e.u = shifted<sizeof(T)>(raw[0], raw[1], off);
        uint32_t w[8] = {e.u.x, e.u.y, e.u.z, e.u.w};
        if constexpr (kWords == 8) {
            e.v = shifted<sizeof(T)>(raw[1], raw[2], off);
            w[4] = e.v.x, w[5] = e.v.y, w[6] = e.v.z, w[7] = e.v.w;
        }
        if (count < 8) {
            constexpr int kPer = 4 / sizeof(T);
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                if (i * kPer >= count) w[i] = 0u;
                else if (kPer == 2 && i * kPer + 1 == count) w[i] &= 0xffffu;
            }
        }
        e.u = make_uint4(w[0], w[1], w[2], w[3]);
        if constexpr (kWords == 8) e.v = make_uint4(w[4], w[5], w[6], w[7]);
        return e;
    }
};

template <typename T, bool WHOLE>
__global__ void __launch_bounds__(256) pack_kernel(PackArgs a, uint32_t strips_per_row, uint32_t strips) {
    const int lane = threadIdx.x & 15;
    const uint32_t q = blockIdx.x * 16 + (threadIdx.x >> 4);
    const bool on = q < strips;                            // the warp's other half may still have work
    const uint32_t r = on ? q / strips_per_row : 0;
    const int blk = (int)(on ? q - r * strips_per_row : 0) * kStrip, col = blk * kBlock + lane * 8;
    const int cols = (int)a.cols;
    const uint32_t g = r / (uint32_t)a.n;
    const int64_t group = g, row = r - g * (uint32_t)a.n;
    const T *x = static_cast<const T *>(a.x.data) + group * a.x.group + row * a.x.row + col;
    uint8_t *codes = static_cast<uint8_t *>(a.codes.data) + group * a.codes.group + row * a.codes.row + col;
    float *scales = static_cast<float *>(a.scales.data) + group * a.scales.group + row * a.scales.row + blk;
    Eight e[kStrip];
#pragma unroll
    for (int i = 0; i < kStrip; ++i) {
        e[i].u = e[i].v = make_uint4(0u, 0u, 0u, 0u);
        if (WHOLE && on && col + i * kBlock < cols) e[i].load(x + i * kBlock);
    }
    if constexpr (!WHOLE) {
        const T *group_x = static_cast<const T *>(a.x.data) + group * a.x.group;
        const uintptr_t from = reinterpret_cast<uintptr_t>(group_x), to = reinterpret_cast<uintptr_t>(group_x + (a.n - 1) * a.x.row + cols);
        Shifted<T> s[kStrip];
#pragma unroll
        for (int i = 0; i < kStrip; ++i) s[i].load(x + i * kBlock, on ? max(min(cols - col - i * kBlock, 8), 0) : 0, from, to);
#pragma unroll
        for (int i = 0; i < kStrip; ++i) e[i] = s[i].get(on ? max(min(cols - col - i * kBlock, 8), 0) : 0);
    }
    // The blocks' largest magnitudes over the 16 lanes: lanes give half of the blocks away at a time until each has one block left
    static_assert(kStrip == 4, "two steps halve the blocks");
    uint32_t most[kStrip];
    unsigned odd = 0;                                      // blocks with an infinity or NaN among the lane's
#pragma unroll
    for (int i = 0; i < kStrip; ++i) {
        most[i] = e[i].most(T());
        if (most[i] >= 0x7f800000u) {
            odd |= 1u << i;
            Two f[4];
            e[i].get(f, T());
            most[i] = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) most[i] = max(most[i], max(finite_bits(f[k].x), finite_bits(f[k].y)));
        }
    }
    const bool upper = lane & 8, second = lane & 4;
    const uint32_t k0 = upper ? most[2] : most[0], k1 = upper ? most[3] : most[1], g0 = upper ? most[0] : most[2], g1 = upper ? most[1] : most[3];
    const uint32_t h0 = max(k0, __shfl_xor_sync(0xffffffffu, g0, 8)), h1 = max(k1, __shfl_xor_sync(0xffffffffu, g1, 8));
    uint32_t amax = max(second ? h1 : h0, __shfl_xor_sync(0xffffffffu, second ? h0 : h1, 4));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    const int mine = amax ? scale_exponent(amax) : 0;      // block lane / 4
    if (on && lane % 4 == 0 && col - lane * 8 + lane / 4 * kBlock < cols) scales[lane / 4] = __uint_as_float((uint32_t)(127 + mine) << 23);
    const uint32_t inv_bits = (uint32_t)(127 - mine) << 23;
#pragma unroll
    for (int i = 0; i < kStrip; ++i) {
        const Two inv = both(__uint_as_float(__shfl_sync(0xffffffffu, inv_bits, i * 4, 16)));
        Two f[4];
        e[i].get(f, T());
        if (on && col + i * kBlock < cols) {
            uint32_t w[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const Two v = mul2(f[h], inv);
                w[h] = __nv_cvt_float2_to_fp8x2(make_float2(v.x, v.y), __NV_SATFINITE, __NV_E4M3);
                if (odd >> i & 1) {                        // infinities saturate in the conversion; they are kept as NaN
                    if (!(fabsf(f[h].x) < INFINITY)) w[h] |= 0x7fu;
                    if (!(fabsf(f[h].y) < INFINITY)) w[h] |= 0x7f00u;
                }
            }
            const uint2 c = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
            if (WHOLE || col + i * kBlock + 8 <= cols) *reinterpret_cast<uint2 *>(codes + i * kBlock) = c;
            else
#pragma unroll
                for (int h = 0; h < 7; ++h)
                    if (col + i * kBlock + h < cols) codes[i * kBlock + h] = (uint8_t)((h < 4 ? c.x : c.y) >> (h % 4 * 8));
        }
    }
}

// dW of a tile of 64 outputs by 64 inputs of one group in a block: ROWS rows at a time through shared memory, the next ones on their way into
// registers, 4 x 4 sums a thread; db with the first tile of the inputs.  For what is over before the tensor cores' kernels have started, and for
// codes that no tensor map can step through (12 groups of 37 rows, 301 x 131: 6 us beside the launch; it reaches about 27 TFLOP/s).
// LONG: sums of more than kChain rows.
constexpr int kChain = 1024;
template <typename T, typename P, int ROWS, bool LONG>
__global__ void __launch_bounds__(256) dense_any_kernel(DenseGradArgs a) {
    constexpr int kTile = 64, kEach = ROWS * kTile / 256, kApart = ROWS / kEach;
    __shared__ __align__(16) float sd[ROWS][kTile], sx[ROWS][kTile];
    const int64_t o0 = (int64_t)blockIdx.y * kTile, k0 = (int64_t)blockIdx.x * kTile;
    const int i = blockIdx.z, tx = threadIdx.x & 15, ty = threadIdx.x >> 4, c = threadIdx.x % kTile, t = threadIdx.x / kTile;
    const bool has_o = o0 + c < a.outputs, has_k = k0 + c < a.inputs;
    const T *dy = static_cast<const T *>(a.dy.data) + i * a.dy.group + o0 + c;
    const uint8_t *codes = static_cast<const uint8_t *>(a.codes.data) + i * a.codes.group + k0 + c;
    const float *scales = static_cast<const float *>(a.scales.data) + i * a.scales.group + (k0 + c) / kBlock;
    float acc[4][4] = {}, bias = 0.f, scale[kEach];
    T d[kEach];
    uint8_t code[kEach];
    auto fetch = [&](int64_t t0) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int64_t row = t0 + t + e * kApart;
            if (row >= a.n) break;
            if (has_o) d[e] = dy[row * a.dy.row];
            if (has_k) {
                code[e] = codes[row * a.codes.row];
                scale[e] = scales[row * a.scales.row];
            }
        }
    };
    LongSum long_acc[LONG ? 4 : 1][LONG ? 4 : 1], long_bias;
    fetch(0);
    for (int64_t t0 = 0; t0 < a.n; t0 += ROWS) {
        if (LONG && t0 % kChain == 0) {
            long_bias.add(bias);
            bias = 0.f;
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    long_acc[LONG ? p : 0][LONG ? q : 0].add(acc[p][q]);
                    acc[p][q] = 0.f;
                }
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const bool on = t0 + t + e * kApart < a.n;
            sd[t + e * kApart][c] = on && has_o ? value_of(&d[e]) : 0.f;
            sx[t + e * kApart][c] = on && has_k ? saved_value(code[e], scale[e]) : 0.f;
        }
        __syncthreads();
        fetch(t0 + ROWS);
        if (a.db && blockIdx.x == 0 && threadIdx.x < kTile)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) bias += sd[r][threadIdx.x];
#pragma unroll 8
        for (int r = 0; r < ROWS; ++r) {
            const float4 dr = *reinterpret_cast<const float4 *>(&sd[r][4 * ty]), xr = *reinterpret_cast<const float4 *>(&sx[r][4 * tx]);
            const float df[4] = {dr.x, dr.y, dr.z, dr.w}, xf[4] = {xr.x, xr.y, xr.z, xr.w};
#pragma unroll
            for (int p = 0; p < 4; ++p)
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[p][q] = fmaf(df[p], xf[q], acc[p][q]);
        }
        __syncthreads();
    }
    if constexpr (LONG) {
        long_bias.add(bias);
        bias = long_bias.sum;
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                long_acc[p][q].add(acc[p][q]);
                acc[p][q] = long_acc[p][q].sum;
            }
    }
    P *dw = static_cast<P *>(a.dw) + i * a.ldw;
    // through shared memory, ROWS outputs at a time, so that a warp writes a row's entries side by side
    float (*out)[kTile] = sd;
#pragma unroll
    for (int part = 0; part < kTile / ROWS; ++part) {
        if (ty / (ROWS / 4) == part)
#pragma unroll
            for (int p = 0; p < 4; ++p)
                *reinterpret_cast<float4 *>(&out[4 * (ty % (ROWS / 4)) + p][4 * tx]) = make_float4(acc[p][0], acc[p][1], acc[p][2], acc[p][3]);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int64_t o = o0 + part * ROWS + t + e * kApart;
            if (o < a.outputs && has_k) put(dw + o * a.inputs + k0 + c, out[t + e * kApart][c]);
        }
        __syncthreads();
    }
    if (a.db && blockIdx.x == 0 && threadIdx.x < kTile && has_o) put(static_cast<P *>(a.db) + i * a.ldb + o0 + threadIdx.x, bias);
}

// db: a cluster takes 32 N outputs of a group, its blocks and their warps the rows in turn, a lane N neighbouring outputs; the warps' sums are
// joined in shared memory, the blocks' through the cluster's.
constexpr int kBiasWarps = 8;
template <typename T, typename P, int N, bool LONG>
__global__ void __launch_bounds__(kBiasWarps * 32) dense_bias_kernel(DenseGradArgs a, int cluster) {
    __shared__ float sums[kBiasWarps][32 * N + 1];
    __shared__ float total[32 * N];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.z, rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int64_t o0 = (int64_t)blockIdx.y * 32 * N, o = o0 + lane * N;
    const T *dy = static_cast<const T *>(a.dy.data) + i * a.dy.group + o;
    float s[N];
    LongSum long_s[LONG ? N : 1];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = 0.f;
    if (o < a.outputs) {
        constexpr int kAtOnce = 8;                               // rows' loads in flight
        const int64_t step = cluster * kBiasWarps;
        int terms = 0;
        for (int64_t t = rank * kBiasWarps + warp; t < a.n; t += kAtOnce * step) {
            if (LONG && terms == kChain) {
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    long_s[LONG ? k : 0].add(s[k]);
                    s[k] = 0.f;
                }
                terms = 0;
            }
            terms += kAtOnce;
            alignas(16) T e[kAtOnce][N];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
                if (t + u * step < a.n) {
                    if constexpr (N * sizeof(T) == 16) *reinterpret_cast<uint4 *>(e[u]) = __ldg(reinterpret_cast<const uint4 *>(dy + (t + u * step) * a.dy.row));
                    else e[u][0] = dy[(t + u * step) * a.dy.row];
                }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u)
                if (t + u * step < a.n)
#pragma unroll
                    for (int k = 0; k < N; ++k) s[k] += value_of(&e[u][k]);
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (LONG) long_s[LONG ? k : 0].add(s[k]);
        sums[warp][k * 32 + lane] = LONG ? long_s[LONG ? k : 0].sum : s[k];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 32 * N; c += kBiasWarps * 32) {
        float v = 0.f;
#pragma unroll
        for (int q = 0; q < kBiasWarps; ++q) v += sums[q][c];
        total[c] = v;
    }
    if (cluster > 1) cluster_barrier();
    if (rank == 0)
        for (int c = threadIdx.x; c < 32 * N; c += kBiasWarps * 32) {
            float v = total[c];
            for (int q = 1; q < cluster; ++q) v += cluster_load(cluster_addr(&total[c], q));
            const int64_t to = o0 + (c & 31) * N + c / 32;
            if (to < a.outputs) put(static_cast<P *>(a.db) + i * a.ldb + to, v);
        }
    if (cluster > 1) cluster_barrier();
    pdl_wait();        // nothing here needs what went before; what comes after needs both
}

template <typename T, typename P, int N>
cudaError_t dense_bias(const DenseGradArgs &a, int cluster, cudaStream_t s) {
    const dim3 grid(cluster, (unsigned)((a.outputs + 32 * N - 1) / (32 * N)), a.m);
    auto *kernel = a.n > (int64_t)kChain * kBiasWarps * cluster ? dense_bias_kernel<T, P, N, true> : dense_bias_kernel<T, P, N, false>;
    if (cluster == 1) return launch_chained(kernel, grid, dim3(kBiasWarps * 32), 0, s, true, a, cluster);
    return launch_clustered(kernel, cluster, grid, dim3(kBiasWarps * 32), 0, s, true, a, cluster);
}

// 16 bytes of outputs a lane where that still gives every SM a block
template <typename T, typename P>
cudaError_t dense_bias(const DenseGradArgs &a, cudaStream_t s) {
    constexpr int N = 16 / sizeof(T);
    int cluster = 1;
    while (cluster < 8 && a.n > cluster * 64) cluster *= 2;          // eight rows a warp and more
    const bool many = (a.outputs + 32 * N - 1) / (32 * N) * a.m * cluster >= 148;
    return many && a.outputs % N == 0 && aligned_to(a.dy, a.m, a.n, sizeof(T), 16) ? dense_bias<T, P, N>(a, cluster, s) : dense_bias<T, P, 1>(a, cluster, s);
}

// Few rows of few tiles are over on the CUDA cores, in one launch, before the tensor cores' launches are.  Beside what any launch costs, as many tiles
// as are resident take about 3 us there for every 32 rows (2 for the only 16); the tensor cores' kernel and the sums of dY 9 us, with dY's terms 13
// and more (12 groups of 37 rows, 301 x 131: 6 us against 17 in binary32; 8 groups of 200 rows, 304 x 304: 22 against 19).
bool dense_on_tensor_cores(int type, const DenseGradArgs &a) {
    const int64_t tiles = (a.inputs + 63) / 64 * ((a.outputs + 63) / 64) * a.m, waves = (tiles + 443) / 444;
    const bool as_it_lies = type == ZENO_BF16 && aligned_to(a.dy, a.m, a.n, 2, 16);
    return waves * (a.n <= 16 ? 2 : (a.n + 31) / 32 * 3) > (as_it_lies ? 8 : 12);
}

template <typename T, typename P>
cudaError_t dense_gradient(int type, int param_type, const DenseGradArgs &a, cudaStream_t s) {
    cudaError_t e = dense_on_tensor_cores(type, a) ? launch_dense_tc(type, param_type, a, s) : cudaErrorNotSupported;
    if (e == cudaErrorNotSupported)
        return launch_chained(a.n <= 16 ? dense_any_kernel<T, P, 16, false> : a.n <= kChain ? dense_any_kernel<T, P, 32, false> : dense_any_kernel<T, P, 32, true>, dim3((unsigned)((a.inputs + 63) / 64), (unsigned)((a.outputs + 63) / 64), a.m), dim3(256), 0, s, false, a);
    return e == cudaSuccess && a.db ? dense_bias<T, P>(a, s) : e;
}

}  // namespace

cudaError_t launch_pack(int type, const PackArgs &a, cudaStream_t s) {
    const int64_t per_row = (a.cols + kBlock - 1) / kBlock;
    const bool whole = a.cols % 8 == 0 && aligned_to(a.x, a.m, a.n, type == ZENO_BF16 ? 2 : 4, 16);
    const int64_t strips_per_row = (per_row + kStrip - 1) / kStrip, strips = strips_per_row * a.m * a.n, grid = (strips + 15) / 16;
    if (aligned_to(a.codes, a.m, a.n, 1, 8) && strips < (int64_t)1 << 31) {
        auto *kernel = type == ZENO_BF16 ? (whole ? pack_kernel<__nv_bfloat16, true> : pack_kernel<__nv_bfloat16, false>)
                                         : (whole ? pack_kernel<float, true> : pack_kernel<float, false>);
        return launch_chained(kernel, dim3((unsigned)grid), dim3(256), 0, s, false, a, (uint32_t)strips_per_row, (uint32_t)strips);
    }
    const int64_t blocks = per_row * a.m * a.n;
    const unsigned any_grid = (unsigned)min((blocks + 7) / 8, (int64_t)148 * 8);
    return launch_chained(type == ZENO_BF16 ? pack_any_kernel<__nv_bfloat16> : pack_any_kernel<float>, dim3(any_grid), dim3(256), 0, s, false, a,
                          per_row, blocks);
}

int64_t dense_gradient_workspace(int type, const DenseGradArgs &a) { return dense_on_tensor_cores(type, a) ? dense_tc_workspace(type, a) : 0; }

cudaError_t launch_dense_gradient(int type, int param_type, const DenseGradArgs &a, cudaStream_t s) {
    if (type == ZENO_BF16)
        return param_type == ZENO_BF16 ? dense_gradient<__nv_bfloat16, __nv_bfloat16>(type, param_type, a, s) : dense_gradient<__nv_bfloat16, float>(type, param_type, a, s);
    return param_type == ZENO_BF16 ? dense_gradient<float, __nv_bfloat16>(type, param_type, a, s) : dense_gradient<float, float>(type, param_type, a, s);
}

}  // namespace zeno

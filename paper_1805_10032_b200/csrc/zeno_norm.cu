// Layer norm of rows of activations, and its backward pass with the weight gradients reduced per group (worker).
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

template <typename T, typename P>
cudaError_t layer_norm(const NormArgs &a, cudaStream_t s) {
    return launch_chained(norm_any_kernel<T, P>, dim3((unsigned)(a.m * a.n)), dim3(kThreads), 0, s, false, a);
}

template <typename T, typename P>
cudaError_t layer_norm_gradient(const NormGradArgs &a, cudaStream_t s) {
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

int64_t norm_gradient_workspace(int m, int64_t n, int64_t cols) { return 0; }

cudaError_t launch_layer_norm_gradient(int type, int param_type, const NormGradArgs &a, cudaStream_t s) {
    if (type == ZENO_BF16)
        return param_type == ZENO_BF16 ? layer_norm_gradient<__nv_bfloat16, __nv_bfloat16>(a, s) : layer_norm_gradient<__nv_bfloat16, float>(a, s);
    return param_type == ZENO_BF16 ? layer_norm_gradient<float, __nv_bfloat16>(a, s) : layer_norm_gradient<float, float>(a, s);
}

}  // namespace zeno

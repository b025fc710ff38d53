// Internal declarations of the language model operators (zeno_norm.cu, zeno_saved.cu, zeno_tokens.cu): arguments checked, the
// device current, at least one row unless noted.
#pragma once

#include "zeno_internal.h"

namespace zeno {

// Rows of m groups of n: row r is row r % n of group r / n.  Strides in elements.
struct Rows {
    void *data;
    int64_t row, group;
    int64_t n;
#ifdef __CUDACC__
    __device__ __forceinline__ int64_t at(int64_t r) const {
        const uint32_t g = (uint32_t)r / (uint32_t)n;          // rows are counted in 31 bits
        return (int64_t)g * group + (int64_t)((uint32_t)r - g * (uint32_t)n) * row;
    }
#endif
};

// Whether every row starts at a multiple of `to` bytes.
inline bool aligned_to(const Rows &v, int m, int64_t n, size_t elem, size_t to) {
    return reinterpret_cast<uintptr_t>(v.data) % to == 0 && (n <= 1 || v.row * elem % to == 0) && (m <= 1 || v.group * elem % to == 0);
}

// The 16 bytes that start `off` bytes into a and end in b (off: 0 .. 14; a multiple of ALIGN, 2 or 4).
template <int ALIGN>
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, unsigned off) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 6; ++i)
        if (off & 8) w[i] = w[i + 2];
#pragma unroll
    for (int i = 0; i < 5; ++i)
        if (off & 4) w[i] = w[i + 1];
    if constexpr (ALIGN == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (off & 2) * 8);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

struct NormArgs {
    Rows x, y;
    int m;
    int64_t n, cols;
    const void *w, *b;
    int64_t ldw;
    float eps;
    float *mean, *rstd;
};
cudaError_t launch_layer_norm(int type, int param_type, const NormArgs &a, cudaStream_t s);

struct NormGradArgs {
    Rows dy, x, codes, scales, dx;      // x.data NULL: codes and scales; dx.data NULL: not wanted
    int m;
    int64_t n, cols;
    const void *w;
    int64_t ldw;
    const float *mean, *rstd;
    void *dw, *db;                      // either may be NULL
    int64_t ldg;
    float *workspace;
};
int64_t norm_gradient_workspace(int m, int64_t n, int64_t cols);
cudaError_t launch_layer_norm_gradient(int type, int param_type, const NormGradArgs &a, cudaStream_t s);   // n may be 0

struct PackArgs {
    Rows x, codes, scales;
    int m;
    int64_t n, cols;
};
cudaError_t launch_pack(int type, const PackArgs &a, cudaStream_t s);

struct DenseGradArgs {
    Rows dy, codes, scales;
    int m;
    int64_t n, inputs, outputs;
    void *dw, *db;                      // db may be NULL
    int64_t ldw, ldb;
    float *workspace;
};
int64_t dense_gradient_workspace(int type, const DenseGradArgs &a);
cudaError_t launch_dense_gradient(int type, int param_type, const DenseGradArgs &a, cudaStream_t s);       // n may be 0

// The same on the tensor cores (zeno_dense_tc.cu), for codes in rows and groups that tensor maps can step through.  NotSupported: it does not
// take the call.  db is not its business.
int64_t dense_tc_workspace(int type, const DenseGradArgs &a);
cudaError_t launch_dense_tc(int type, int param_type, const DenseGradArgs &a, cudaStream_t s);
void set_operator_wait_limit(uint32_t polls);
cudaError_t read_operator_status(int device, cudaStream_t s, int *status);

struct LogprobArgs {
    Rows logits;
    int m;
    int64_t n, vocab;
    const int32_t *targets;
    int top;
    float *logprobs, *entropy, *lse;
    int32_t *top_idx;
    float *top_logprobs;
    int long_sums;                      // by the definition, whose sums may have any number of terms; the launch sets it
};
cudaError_t launch_token_logprobs(int type, const LogprobArgs &a, cudaStream_t s);

struct TokenGradArgs {
    Rows logits, grad;
    int m;
    int64_t n, vocab;
    const int32_t *targets;
    const float *lse, *entropy, *g_logprob, *g_entropy;
};
cudaError_t launch_token_gradient(int type, const TokenGradArgs &a, cudaStream_t s);

#ifdef __CUDACC__

// An element as it lies in memory; without the read-only path, since an output may lie in its input's place.
__device__ __forceinline__ float value_of(const float *p) { return *p; }
__device__ __forceinline__ float value_of(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

// Sum over the block in every thread; `scratch` holds a float for each warp and may be used again after the next barrier.
template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float *scratch) {
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) s += scratch[i];
    return s;
}

// A sum of sums, each of kShortSum terms or a few more, with what its additions lose given back to the next term (Kahan, Further remarks on reducing
// truncation errors, 1965): however many there are, it is off by little more than they are.  By one chain of additions 2^18 equal terms come out wrong
// by up to a hundredth.
constexpr int kShortSum = 64;
struct LongSum {
    float sum = 0.f, lost = 0.f;
    __device__ __forceinline__ void add(float v) {
        const float y = __fsub_rn(v, lost), t = __fadd_rn(sum, y);
        lost = __fsub_rn(__fsub_rn(t, sum), y);
        if (!(fabsf(lost) < INFINITY)) lost = 0.f;          // the sum is not finite
        sum = t;
    }
};

// Two binary32 numbers that one instruction takes
struct Two { float x, y; };
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two d;
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two d;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two d;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ Two both(float v) { return Two{v, v}; }

#endif

}  // namespace zeno

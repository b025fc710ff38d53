// Log probabilities of given tokens with entropy and top alternatives, and their gradient at the logits.
#include "zeno_operators.h"

namespace zeno {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
// exp is zero in binary32 below this: a logarithm under it may be taken as it, so that zero times it is zero
constexpr float kLogOfNothing = -200.f;

template <typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V *scratch, F op) {
#pragma unroll
    for (int s = 16; s >= 1; s >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, s));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int i = 1; i < kThreads / 32; ++i) v = op(v, scratch[i]);
    return v;
}

// What a row's statistics say of a logit: with the largest logit m and S = sum exp(z - m),
// log p = (z - m) - log S.  A row of minus infinities has m = 0 here, S = 0.
__device__ __forceinline__ float log_prob(float z, float m, float log_s) { return log_s == -INFINITY ? -INFINITY : (z - m) - log_s; }

// A block takes a row: its maximum, then the sums, then one maximum after another in the order of their keys.
template <typename T>
__global__ void __launch_bounds__(kThreads) logprobs_any_kernel(LogprobArgs a) {
    __shared__ float scratch[kThreads / 32];
    __shared__ unsigned long long keys[kThreads / 32];
    const int64_t r = blockIdx.x;
    const T *z = static_cast<const T *>(a.logits.data) + a.logits.at(r);
    float m = -INFINITY;
    for (int64_t j = threadIdx.x; j < a.vocab; j += kThreads) m = fmaxf(m, value_of(z + j));
    m = block_reduce(m, scratch, [](float p, float q) { return fmaxf(p, q); });
    if (m == -INFINITY) m = 0.f;
    float s = 0.f, e = 0.f;
    for (int64_t j = threadIdx.x; j < a.vocab; j += kThreads) {
        const float d = value_of(z + j) - m, p = exp2f(d * kLog2e);
        s += p;
        e = fmaf(p, fmaxf(d, kLogOfNothing), e);
    }
    auto add = [](float p, float q) { return p + q; };
    s = block_reduce(s, scratch, add);
    e = block_reduce(e, scratch, add);
    const float log_s = logf(s);
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[r] = m + log_s;
        if (a.entropy) a.entropy[r] = s == 0.f ? 0.f : log_s - e / s;
        if (a.logprobs) {
            const int t = a.targets[r];
            a.logprobs[r] = t >= 0 && t < a.vocab ? log_prob(value_of(z + t), m, log_s) : 0.f;
        }
    }
    unsigned long long below = ~0ull;
    for (int k = 0; k < a.top; ++k) {
        unsigned long long best = 0;
        for (int64_t j = threadIdx.x; j < a.vocab; j += kThreads) {
            const unsigned long long key = rank_key(value_of(z + j), (int)j);
            if (key < below && key > best) best = key;
        }
        below = block_reduce(best, keys, [](unsigned long long p, unsigned long long q) { return p > q ? p : q; });
        if (threadIdx.x == 0) {
            const int j = (int)(0xffffffffu - (uint32_t)below);
            if (a.top_idx) a.top_idx[r * a.top + k] = j;
            if (a.top_logprobs) a.top_logprobs[r * a.top + k] = log_prob(value_of(z + j), m, log_s);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) token_gradient_any_kernel(TokenGradArgs a) {
    const int64_t r = blockIdx.x;
    const T *z = static_cast<const T *>(a.logits.data) + a.logits.at(r);
    T *out = static_cast<T *>(a.grad.data) + a.grad.at(r);
    const int t = a.targets[r];
    const bool given = t >= 0 && t < a.vocab;
    const float lse = a.lse[r], g = given ? a.g_logprob[r] : 0.f, h = a.g_entropy ? a.g_entropy[r] : 0.f;
    const float entropy = a.g_entropy ? a.entropy[r] : 0.f;
    if ((!given && !a.g_entropy) || lse == -INFINITY) {
        for (int64_t j = threadIdx.x; j < a.vocab; j += kThreads) put(out + j, 0.f);
        return;
    }
    for (int64_t j = threadIdx.x; j < a.vocab; j += kThreads) {
        const float lp = value_of(z + j) - lse, p = exp2f(lp * kLog2e);
        // p (g + h (log p + H)), whose second factor stays finite where p is zero
        const float v = (j == t && given ? g : 0.f) - p * fmaf(h, fmaxf(lp, kLogOfNothing) + entropy, g);
        put(out + j, v);
    }
}

}  // namespace

cudaError_t launch_token_logprobs(int type, const LogprobArgs &a, cudaStream_t s) {
    return launch_chained(type == ZENO_BF16 ? logprobs_any_kernel<__nv_bfloat16> : logprobs_any_kernel<float>, dim3((unsigned)(a.m * a.n)),
                          dim3(kThreads), 0, s, false, a);
}

cudaError_t launch_token_gradient(int type, const TokenGradArgs &a, cudaStream_t s) {
    return launch_chained(type == ZENO_BF16 ? token_gradient_any_kernel<__nv_bfloat16> : token_gradient_any_kernel<float>, dim3((unsigned)(a.m * a.n)),
                          dim3(kThreads), 0, s, false, a);
}

}  // namespace zeno

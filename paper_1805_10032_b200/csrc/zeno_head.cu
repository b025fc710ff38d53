// Log probabilities of given tokens from the last hidden states and the output layer's weights, piece by piece of the vocabulary and without keeping
// logits, and their gradient:
//   z = scale x W^T,  lse = log sum_j exp(z_j),  logprob = z_target - lse;
//   D_tj = g_t scale ([j = target] - exp(z_tj - lse_t)),  dx = D W,  dW = D^T x (every worker's own).
// Tokens without a target take no part: the others are gathered into slots first (their hidden states as bfloat16 terms, one of a bfloat16 number and three of a
// binary32 one), each worker's in a run of its own that empty slots fill up to a multiple of kSlots, so that a worker's dW is a sum over whole stages.
// Weights that no tensor copy can step through, and binary32 ones, are rewritten in terms a piece at a time.
#include "zeno_head.h"

namespace zeno {

namespace {

constexpr int64_t kPieceBytes = (int64_t)128 << 20, kWeightBytes = (int64_t)256 << 20;
constexpr int kMinPiece = 2048;

// What lies where in the workspace, and how the vocabulary is cut.
struct Plan {
    int x_terms, w_terms, w_packed, prob_terms, groups, splits, pieces;
    int64_t group_slots, slots, pitch, piece, parts_pitch, part_pitch;
    int64_t counts, begin, end, total, list, rank, target, lse, g, target_logit, x, w, part, probs, parts, bytes;
};

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

bool mappable(const void *w, int64_t ldw, int64_t groups, int64_t cols) {
    const int64_t limit = (int64_t)1 << 39;
    return reinterpret_cast<uintptr_t>(w) % 16 == 0 && cols % 8 == 0 && (groups <= 1 || (ldw % 8 == 0 && ldw < limit));
}

Plan plan_head(int type, int param_type, bool gradient, const HeadArgs &a) {
    Plan p = {};
    p.groups = a.ldw != 0 && a.m > 1 ? a.m : 1;
    p.x_terms = type == ZENO_F32 ? 3 : 1;
    p.w_terms = param_type == ZENO_F32 ? 3 : 1;
    p.w_packed = p.w_terms > 1 || !mappable(a.w, a.ldw, p.groups, a.cols);
    p.prob_terms = p.x_terms > 1 || p.w_terms > 1 ? 3 : 1;
    // groups whose tiles of rows are written whole must not share one
    const int64_t worker_slots = up(a.n, p.groups > 1 && gradient ? 256 : kSlots);
    p.slots = worker_slots * a.m;
    p.group_slots = p.groups > 1 ? worker_slots : p.slots;
    p.pitch = up(a.cols, 8);
    p.parts_pitch = up(a.cols, 4);
    const int64_t per_word = p.w_packed ? p.groups * p.w_terms * p.pitch * 2 : 0, per_prob = gradient ? p.slots * p.prob_terms * 2 : 0;
    int64_t most = a.vocab;
    if (per_word && kWeightBytes / per_word < most) most = kWeightBytes / per_word;
    if (per_prob && kPieceBytes / per_prob < most) most = kPieceBytes / per_prob;
    if (most < kMinPiece) most = kMinPiece;
    p.pieces = (int)((a.vocab + most - 1) / most);
    p.piece = up((a.vocab + p.pieces - 1) / p.pieces, 256);
    p.pieces = (int)((a.vocab + p.piece - 1) / p.piece);
    p.splits = 1;
    if (gradient) {
        // few tiles of dx: the words are cut, and the parts joined
        const int64_t tiles = up(p.group_slots, 256) / 256 * (up(a.cols, 256) / 256) * p.groups, stages = p.piece / 64;
        int64_t splits = 74 / (tiles > 0 ? tiles : 1);
        if (splits > stages / 8) splits = stages / 8;
        p.splits = splits < 1 ? 1 : (int)splits;
    }
    p.part_pitch = up(a.vocab, 256) / 128;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t from = at;
        at += up(bytes, 256);
        return from;
    };
    p.counts = take(a.m * 4);
    p.begin = take(a.m * 4);
    p.end = take(a.m * 4);
    p.total = take(8);
    p.list = take(a.m * a.n * 4);
    p.rank = take(a.m * a.n * 4);
    p.target = take(p.slots * 4);
    p.lse = take(gradient ? p.slots * 4 : 0);
    p.g = take(gradient ? p.slots * 4 : 0);
    p.target_logit = take(gradient ? 0 : p.slots * 4);
    p.x = take(p.x_terms * p.slots * p.pitch * 2);
    p.w = take(per_word * p.piece);
    p.part = take(gradient ? 0 : p.slots * p.part_pitch * 8);
    p.probs = take(p.piece * per_prob);
    p.parts = take(gradient && a.dx.data ? p.splits * p.slots * p.parts_pitch * 4 : 0);
    p.bytes = at;
    return p;
}

// ---- tokens to slots

constexpr int kOrderThreads = 512;

// A worker's tokens that carry a target, in their order: list[worker][k] is the k-th one, rank[worker][token] its k or -1.
__global__ void __launch_bounds__(kOrderThreads) head_order_kernel(const int32_t *targets, int64_t n, int64_t vocab, int *counts, int *list, int *rank) {
    __shared__ int warp_count[kOrderThreads / 32];
    pdl_wait();
    pdl_launch_dependents();
    const int worker = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    targets += worker * n;
    list += worker * n;
    rank += worker * n;
    int base = 0;
    for (int64_t t0 = 0; t0 < n; t0 += kOrderThreads) {
        const int64_t t = t0 + threadIdx.x;
        const bool given = t < n && (uint32_t)targets[t] < (uint64_t)vocab;
        const unsigned votes = __ballot_sync(0xffffffffu, given);
        if (lane == 0) warp_count[warp] = __popc(votes);
        __syncthreads();
        int before = base, all = 0;
#pragma unroll
        for (int w = 0; w < kOrderThreads / 32; ++w) {
            if (w < warp) before += warp_count[w];
            all += warp_count[w];
        }
        const int k = before + __popc(votes & ((1u << lane) - 1));
        if (given) list[k] = (int)t;
        if (t < n) rank[t] = given ? k : -1;
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) counts[worker] = base;
}

// The leading 8 bits of what is left of each number, TERMS times: three hold a binary32 number exactly (from 2^-110 on; a smaller one has bits under
// bfloat16's smallest step, 2^-133).  An infinity or NaN is its first term.
template <int TERMS>
__device__ __forceinline__ void put_terms(float (&f)[8], __nv_bfloat16 *to, int64_t plane) {
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
        alignas(16) __nv_bfloat16 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            v[k] = __float2bfloat16_rn(f[k]);
            if (TERMS > 1) {
                // (a finite number may round to infinity: then the term is the largest finite one)
                if (fabsf(f[k]) < INFINITY && !(fabsf(__bfloat162float(v[k])) < INFINITY)) v[k] = __ushort_as_bfloat16(f[k] < 0.f ? 0xff7f : 0x7f7f);
                f[k] = fabsf(f[k]) < INFINITY ? f[k] - __bfloat162float(v[k]) : 0.f;
            }
        }
        *reinterpret_cast<uint4 *>(to + t * plane) = *reinterpret_cast<const uint4 *>(v);
    }
}

// A warp rewrites a row of cols entries (NULL: zeros), eight to a lane.
template <typename T, int TERMS>
__device__ __forceinline__ void row_terms(const T *from, int64_t cols, int64_t pitch, __nv_bfloat16 *to, int64_t plane, bool vectors) {
    for (int64_t c = (threadIdx.x & 31) * 8; c < pitch; c += 256) {
        float f[8] = {};
        if (from && vectors) {
            alignas(16) T e[8];
#pragma unroll
            for (int k = 0; k < (int)sizeof(e) / 16; ++k) reinterpret_cast<uint4 *>(e)[k] = reinterpret_cast<const uint4 *>(from + c)[k];
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = value_of(e + k);
        } else if (from) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < cols) f[k] = value_of(from + c + k);
        }
        put_terms<TERMS>(f, to + c, plane);
    }
}

struct SlotsArgs {
    HeadArgs a;
    Plan p;
    int vectors;
};

template <typename V>
__host__ __device__ __forceinline__ V *at(const HeadArgs &a, int64_t offset) {
    return reinterpret_cast<V *>(static_cast<uint8_t *>(a.workspace) + offset);
}

// A warp per slot: blockIdx.y is the worker.
template <typename T, int TERMS>
__global__ void __launch_bounds__(256) head_slots_kernel(const SlotsArgs args) {
    __shared__ int scratch[8];
    const HeadArgs &a = args.a;
    const Plan &p = args.p;
    pdl_wait();
    pdl_launch_dependents();
    const int worker = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int *counts = at<int>(a, p.counts);
    const int count = counts[worker], filled = (count + kSlots - 1) / kSlots * kSlots;
    int begin = 0;
    if (p.groups > 1) {
        begin = (int)(worker * p.group_slots);
    } else {                                                          // behind the workers before
        for (int i = threadIdx.x; i < worker; i += 256) begin += (counts[i] + kSlots - 1) / kSlots * kSlots;
        begin = __reduce_add_sync(0xffffffffu, begin);
        if (lane == 0) scratch[warp] = begin;
        __syncthreads();
        begin = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) begin += scratch[i];
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        at<int>(a, p.begin)[worker] = begin;
        at<int>(a, p.end)[worker] = begin + filled;
        if (worker == a.m - 1) {
            at<int>(a, p.total)[0] = 0;
            at<int>(a, p.total)[1] = begin + filled;
        }
    }
    for (int k = blockIdx.x * 8 + warp; k < filled; k += gridDim.x * 8) {
        const int token = k < count ? at<int>(a, p.list)[worker * a.n + k] : -1;
        const int64_t slot = begin + k, row = worker * a.n + token;
        if (lane == 0) {
            at<int>(a, p.target)[slot] = token >= 0 ? a.targets[row] : -1;
            if (a.g) {
                at<float>(a, p.lse)[slot] = token >= 0 ? a.lse_in[row] : -INFINITY;
                at<float>(a, p.g)[slot] = token >= 0 ? a.g[row] * a.scale : 0.f;
            }
        }
        const T *from = token >= 0 ? static_cast<const T *>(a.x.data) + worker * a.x.group + token * a.x.row : nullptr;
        row_terms<T, TERMS>(from, a.cols, p.pitch, at<__nv_bfloat16>(a, p.x) + slot * p.pitch, p.slots * p.pitch, args.vectors);
    }
}

// Words v0 .. v0 + words - 1 of every group's weights: [group][term][piece][pitch].  A warp per word.
template <typename T, int TERMS>
__global__ void __launch_bounds__(256) head_words_kernel(const T *w, int64_t ldw, int64_t cols, int64_t pitch, int64_t v0, int words, int64_t piece, int64_t total,
                                                         __nv_bfloat16 *out, int vectors) {
    pdl_wait();
    pdl_launch_dependents();
    for (int64_t q = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); q < total; q += (int64_t)gridDim.x * 8) {
        const int64_t group = q / words, v = q - group * words;
        row_terms<T, TERMS>(w + group * ldw + (v0 + v) * cols, cols, pitch, out + (group * TERMS * piece + v) * pitch, piece * pitch, vectors);
    }
}

// ---- ends (a call's last kernel lets nothing start before its end)

// lse and log probability of every token from its parts of the vocabulary: a warp per token.
__global__ void __launch_bounds__(256) head_join_kernel(const HeadArgs a, const Plan p, int parts) {
    pdl_wait();
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= a.m * a.n) return;
    const int rank = at<int>(a, p.rank)[row];
    float lse = 0.f, logprob = 0.f;
    if (rank >= 0) {
        const int64_t slot = at<int>(a, p.begin)[row / a.n] + rank;
        const float2 *part = at<float2>(a, p.part) + slot * p.part_pitch;
        float most = -INFINITY;
        for (int i = lane; i < parts; i += 32) most = fmaxf(most, part[i].x);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
        const float beside = most == -INFINITY ? 0.f : most;
        double sum = 0.;
        for (int i = lane; i < parts; i += 32) {
            const float2 v = part[i];
            sum += (double)(v.y * (v.x == -INFINITY ? 1.f : expf(v.x - beside)));       // a part of nothing but minus infinity sums to zero, or NaN
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const double log_sum = log(sum);
        lse = (float)(beside + log_sum);
        logprob = sum == 0. ? -INFINITY : (float)((double)at<float>(a, p.target_logit)[slot] - beside - log_sum);
    }
    if (lane == 0) {
        if (a.lse) a.lse[row] = lse;
        if (a.logprobs) a.logprobs[row] = logprob;
    }
}

// dx: the parts' sums, four neighbouring entries a thread, rounded once; zero without a target.
template <typename T>
__global__ void __launch_bounds__(256) head_inputs_kernel(const HeadArgs a, const Plan p, int vectors) {
    pdl_wait();
    const int64_t per_row = p.parts_pitch / 4, total = (int64_t)a.m * a.n * per_row, plane = p.slots * p.parts_pitch;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
        const int64_t row = q / per_row, c = (q - row * per_row) * 4, worker = row / a.n;
        const int rank = at<int>(a, p.rank)[row];
        float s[4] = {};
        if (rank >= 0) {
            const float *from = at<float>(a, p.parts) + (at<int>(a, p.begin)[worker] + rank) * p.parts_pitch + c;
            for (int i = 0; i < p.splits; ++i) {
                const float4 v = *reinterpret_cast<const float4 *>(from + i * plane);
                s[0] += v.x, s[1] += v.y, s[2] += v.z, s[3] += v.w;
            }
        }
        T *to = static_cast<T *>(a.dx.data) + worker * a.dx.group + (row - worker * a.n) * a.dx.row + c;
        alignas(16) T e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) put(e + k, s[k]);
        if (vectors) {
            if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(e);
            else *reinterpret_cast<uint2 *>(to) = *reinterpret_cast<const uint2 *>(e);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (c + k < a.cols) to[k] = e[k];
        }
    }
}

// dW of workers without a single token
template <typename P>
__global__ void __launch_bounds__(256) head_zero_kernel(P *dw, int64_t per_group, int64_t ldw, int64_t total) {
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
        const int64_t group = q / per_group;
        dw[group * ldw + (q - group * per_group)] = P(0.f);
    }
}

dim3 grid_for(int64_t blocks) { return dim3((unsigned)(blocks < 148 * 16 ? blocks : 148 * 16)); }

// Terms that are multiplied: those of the smallest products first.
void set_pairs(HeadTcArgs *h, int a_terms, int b_terms) {
    h->pairs = 0;
    for (int order = 2; order >= 0; --order)
        for (int i = 0; i <= order; ++i)
            if (i < a_terms && order - i < b_terms) {
                h->pair_a[h->pairs] = i;
                h->pair_b[h->pairs++] = order - i;
            }
}

cudaError_t fill_slots(int type, const HeadArgs &a, const Plan &p, cudaStream_t s) {
    cudaError_t e = launch_chained(head_order_kernel, dim3(a.m), dim3(kOrderThreads), 0, s, true, a.targets, a.n, a.vocab, at<int>(a, p.counts), at<int>(a, p.list), at<int>(a, p.rank));
    if (e != cudaSuccess) return e;
    const int elem = type == ZENO_F32 ? 4 : 2;
    const SlotsArgs args = {a, p, a.cols % 8 == 0 && aligned_to(a.x, a.m, a.n, elem, 16)};
    const int64_t blocks = up(a.n, kSlots) / 8;
    const dim3 grid((unsigned)(blocks < 2048 ? blocks : 2048), a.m);
    return type == ZENO_F32 ? launch_chained(head_slots_kernel<float, 3>, grid, dim3(256), 0, s, true, args)
                            : launch_chained(head_slots_kernel<__nv_bfloat16, 1>, grid, dim3(256), 0, s, true, args);
}

// The piece's weights as an operand; rewrites them if they have to be.
cudaError_t piece_weights(int param_type, const HeadArgs &a, const Plan &p, int64_t v0, int64_t words, Operand *o, int64_t *row0, cudaStream_t s) {
    if (!p.w_packed) {
        *o = Operand{a.w, a.cols, a.vocab, a.cols, p.groups > 1 ? a.ldw : a.cols, p.groups};
        *row0 = v0;
        return cudaSuccess;
    }
    *o = Operand{at<void>(a, p.w), a.cols, words, p.pitch, p.piece * p.pitch, p.groups * p.w_terms};
    *row0 = 0;
    const int size = param_type == ZENO_F32 ? 4 : 2;
    const int64_t total = p.groups * words;
    const int vectors = a.cols % 8 == 0 && reinterpret_cast<uintptr_t>(a.w) % 16 == 0 && (p.groups <= 1 || a.ldw * size % 16 == 0);
    auto *out = at<__nv_bfloat16>(a, p.w);
    return param_type == ZENO_F32 ? launch_chained(head_words_kernel<float, 3>, grid_for((total + 7) / 8), dim3(256), 0, s, true, static_cast<const float *>(a.w), a.ldw, a.cols, p.pitch, v0,
                                                   (int)words, p.piece, total, out, vectors)
                                  : launch_chained(head_words_kernel<__nv_bfloat16, 1>, grid_for((total + 7) / 8), dim3(256), 0, s, true, static_cast<const __nv_bfloat16 *>(a.w), a.ldw, a.cols,
                                                   p.pitch, v0, (int)words, p.piece, total, out, vectors);
}

HeadTcArgs common(const HeadArgs &a, const Plan &p, HeadStep step) {
    HeadTcArgs h = {};
    h.step = step;
    h.groups = p.groups;
    h.begin = p.groups > 1 ? at<int>(a, p.begin) : at<int>(a, p.total);
    h.end = p.groups > 1 ? at<int>(a, p.end) : at<int>(a, p.total) + 1;
    h.slots = p.slots;
    h.group_slots = p.group_slots;
    h.cols = a.cols;
    h.vocab = a.vocab;
    h.b_terms = p.w_terms;
    h.scale = a.scale;
    h.targets = at<int>(a, p.target);
    return h;
}

Operand slots_operand(const HeadArgs &a, const Plan &p) { return Operand{at<void>(a, p.x), a.cols, p.slots, p.pitch, p.slots * p.pitch, p.x_terms}; }

}  // namespace

int64_t head_workspace(int type, int param_type, bool gradient, const HeadArgs &a) { return a.m > 0 && a.n > 0 ? plan_head(type, param_type, gradient, a).bytes : 0; }

cudaError_t launch_head_logprobs(int type, int param_type, const HeadArgs &a, cudaStream_t s) {
    const Plan p = plan_head(type, param_type, false, a);
    cudaError_t e = fill_slots(type, a, p, s);
    for (int i = 0; i < p.pieces && e == cudaSuccess; ++i) {
        HeadTcArgs h = common(a, p, HeadStep::kSums);
        h.v0 = i * p.piece;
        h.piece = a.vocab - h.v0 < p.piece ? a.vocab - h.v0 : p.piece;
        e = piece_weights(param_type, a, p, h.v0, h.piece, &h.b, &h.b_row0, s);
        if (e != cudaSuccess) break;
        h.a = slots_operand(a, p);
        set_pairs(&h, p.x_terms, p.w_terms);
        h.part = at<float2>(a, p.part);
        h.part_pitch = p.part_pitch;
        h.target_logit = at<float>(a, p.target_logit);
        e = launch_head_tc(h, s);
    }
    if (e != cudaSuccess) return e;
    return launch_chained(head_join_kernel, dim3((unsigned)((a.m * a.n + 7) / 8)), dim3(256), 0, s, true, a, p, (int)(up(a.vocab, 128) / 128));
}

cudaError_t launch_head_gradient(int type, int param_type, const HeadArgs &a, cudaStream_t s) {
    if (a.n == 0) {
        if (!a.dw) return cudaSuccess;
        const int64_t per_group = a.vocab * a.cols, total = per_group * a.m, blocks = (total + 255) / 256;
        return param_type == ZENO_BF16 ? launch_chained(head_zero_kernel<__nv_bfloat16>, grid_for(blocks), dim3(256), 0, s, false, static_cast<__nv_bfloat16 *>(a.dw), per_group, a.lddw, total)
                                       : launch_chained(head_zero_kernel<float>, grid_for(blocks), dim3(256), 0, s, false, static_cast<float *>(a.dw), per_group, a.lddw, total);
    }
    const Plan p = plan_head(type, param_type, true, a);
    cudaError_t e = fill_slots(type, a, p, s);
    for (int i = 0; i < p.pieces && e == cudaSuccess; ++i) {
        HeadTcArgs h = common(a, p, HeadStep::kProbs);
        h.v0 = i * p.piece;
        h.piece = a.vocab - h.v0 < p.piece ? a.vocab - h.v0 : p.piece;
        Operand w;
        int64_t w_row0;
        e = piece_weights(param_type, a, p, h.v0, h.piece, &w, &w_row0, s);
        if (e != cudaSuccess) break;
        h.a = slots_operand(a, p);
        h.b = w;
        h.b_row0 = w_row0;
        set_pairs(&h, p.x_terms, p.w_terms);
        h.lse = at<float>(a, p.lse);
        h.g = at<float>(a, p.g);
        h.probs = at<__nv_bfloat16>(a, p.probs);
        h.prob_pitch = p.piece;
        h.prob_terms = p.prob_terms;
        e = launch_head_tc(h, s);
        if (e != cudaSuccess) break;
        const Operand probs = {h.probs, h.piece, p.slots, p.piece, p.slots * p.piece, p.prob_terms};
        if (a.dx.data) {
            h.step = HeadStep::kInputs;
            h.a = probs;
            set_pairs(&h, p.prob_terms, p.w_terms);
            h.parts = at<float>(a, p.parts);
            h.parts_pitch = p.parts_pitch;
            h.splits = p.splits;
            h.accumulate = i > 0;
            e = launch_head_tc(h, s);
            if (e != cudaSuccess) break;
        }
        if (a.dw) {
            h.step = HeadStep::kWeights;
            h.a = probs;
            h.b = slots_operand(a, p);
            h.b_row0 = 0;
            set_pairs(&h, p.prob_terms, p.x_terms);
            h.groups = a.m;
            h.begin = at<int>(a, p.begin);
            h.end = at<int>(a, p.end);
            h.dw = a.dw;
            h.lddw = a.lddw;
            h.param_type = param_type;
            h.last = !a.dx.data && i + 1 == p.pieces;
            e = launch_head_tc(h, s);
        }
    }
    if (e != cudaSuccess || !a.dx.data) return e;
    const int size = type == ZENO_F32 ? 4 : 2;
    const int vectors = a.cols % 4 == 0 && aligned_to(a.dx, a.m, a.n, size, 4 * size);
    const int64_t blocks = (a.m * a.n * (p.parts_pitch / 4) + 255) / 256;
    return type == ZENO_F32 ? launch_chained(head_inputs_kernel<float>, grid_for(blocks), dim3(256), 0, s, true, a, p, vectors)
                            : launch_chained(head_inputs_kernel<__nv_bfloat16>, grid_for(blocks), dim3(256), 0, s, true, a, p, vectors);
}

}  // namespace zeno

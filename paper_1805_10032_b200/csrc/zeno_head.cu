// Log probabilities of given tokens from the last hidden states and the output layer's weights, piece by piece of the vocabulary and without keeping
// logits, and their gradient:
//   z = scale x W^T,  lse = log sum_j exp(z_j),  logprob = z_target - lse;
//   D_tj = g_t scale ([j = target] - exp(z_tj - lse_t)),  dx = D W,  dW = D^T x (every worker's own).
// Tokens without a target take no part: the others are gathered into slots first (their hidden states as bfloat16 terms, one of a bfloat16 number and three of a
// binary32 one), each worker's in a run of its own; for the gradient empty slots fill it up to a multiple of kSlots, so that a worker's dW is a sum over whole instructions.
// Weights that no tensor copy can step through, and binary32 ones, are rewritten in terms a piece at a time.
#include "zeno_head.h"

namespace zeno {

namespace {

// Of D, and of rewritten weights.  Every boundary between launches shows: 10 x 1778 tokens, 7744 words by 320 columns (binary32, weights bfloat16) take 1.24 ms,
// in pieces of 256 MB 1.35, of 1 GB 1.17.
constexpr int64_t kPieceBytes = (int64_t)512 << 20, kWeightBytes = (int64_t)768 << 20;
constexpr int kMinPiece = 2048;                                       // words of a piece whatever its bytes (8 x 32768 tokens, 32000 words by 256 columns in bfloat16: 27.1 ms, by 256 42.4)

// What lies where in the workspace, and how the vocabulary is cut.
struct Plan {
    int x_terms, w_terms, w_packed, prob_terms, groups, most_splits, pieces, tile_cols, sum_cols, sum_blocks, sum_words, few, few_blocks, logits_parts, lot;
    int64_t group_slots, slots, pitch, piece, parts_pitch, part_pitch, logits_pitch;
    int64_t counts, begin, end, total, list, rank, target, lse, g, target_logit, x, w, part, probs, parts, extra, bytes;
};

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

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

// Words of a part of lse.
int head_part_words(int tile_cols, int x_terms, int w_terms, int64_t cols) {
    HeadTcArgs h = {};
    set_pairs(&h, x_terms, w_terms);
    return head_brief(h.pairs, cols) ? 64 : tile_cols / 2;
}

bool mappable(const void *w, int64_t ldw, int64_t groups, int64_t cols) {
    const int64_t limit = (int64_t)1 << 39;
    return reinterpret_cast<uintptr_t>(w) % 16 == 0 && cols % 8 == 0 && (groups <= 1 || (ldw % 8 == 0 && ldw < limit));
}

// Few tokens take no tensor cores: the weights go by once for every kFew tokens.  32000 words by 4096 columns, tokens in brackets, here and on the tensor
// cores: bfloat16 62 us (1), 73 (2), 87 (3), there 75 for any number; binary32 hidden states 62 (1), 93 (4), 138 (6), there 128; binary32 weights 101 (1), 128 (4),
// 183 (8), 247 (12), there 452; bfloat16 words that are not aligned, by 4095 columns, 372 (1), there 168.
constexpr int kFew = 4;
constexpr int64_t kFewCols = 8192;                                    // their chains of additions are as long as the tensor cores' stretches
// A warp takes as long for a word of a few columns as for one of 256, some 0.28 ns a word in all, and bfloat16 rows of 1,024 columns as much on their way from
// memory: of many narrow words the tensor cores are quicker once that outweighs their launches (one token of 8 models of 50000 words by 64 columns: 110 us, there
// 46; by 384 116, 81; but of one model by 64 24, 24; by 768 28, 38; 131072 words by 2048 97, 118).  Binary32 weights, four and eight tokens of 8 models of 50000
// words: by 64 columns 153 and 294 us, there 217; by 256 157 and 302, there 332; of 512 by 64 13 and 13, there 18.
constexpr int64_t kNarrow = 1024, kNarrowTimesWords = (int64_t)50 << 20, kNarrowF32 = 256, kManyWordsF32 = 40960;

// Tokens of a group that this way is quicker for; words: of all groups.
int64_t few_tokens(int type, int param_type, bool aligned, int64_t cols, int64_t words) {
    if (param_type == ZENO_F32) return cols < kNarrowF32 && words > kManyWordsF32 ? kFew : 3 * kFew;
    if (!aligned || (cols < kNarrow && (kNarrow - cols) * words > kNarrowTimesWords)) return 0;
    return type == ZENO_F32 ? kFew : 2;
}

Plan plan_head(int type, int param_type, bool gradient, const HeadArgs &a) {
    Plan p = {};
    p.groups = a.ldw != 0 && a.m > 1 ? a.m : 1;
    const int64_t group_rows = p.groups > 1 ? a.n : a.m * a.n;
    p.few = !gradient && a.cols <= kFewCols && group_rows <= few_tokens(type, param_type, mappable(a.w, a.ldw, p.groups, a.cols), a.cols, p.groups * a.vocab);
    if (p.few) {
        const int64_t lots = (group_rows + kFew - 1) / kFew, most = (a.vocab + 15) / 16, blocks = 2 * 2 * kHeadPairs / (p.groups * lots);      // two blocks an SM
        p.few_blocks = (int)(blocks < 1 ? 1 : blocks < most ? blocks : most);
        p.part_pitch = p.few_blocks;
        p.target_logit = 0;
        p.part = up(a.m * a.n * 4, 256);
        p.bytes = p.part + a.m * a.n * p.part_pitch * 8;
        return p;
    }
    p.x_terms = type == ZENO_F32 ? 3 : 1;
    p.w_terms = param_type == ZENO_F32 ? 3 : 1;
    p.w_packed = p.w_terms > 1 || !mappable(a.w, a.ldw, p.groups, a.cols);
    // groups whose tiles of rows are written whole must not share one (as the logits may be, and dx is)
    p.lot = p.groups > 1 || gradient ? kSlots : 1;
    const int64_t worker_slots = up(a.n, p.groups > 1 ? (gradient || a.n > 128 ? 256 : 128) : p.lot);
    p.slots = up(worker_slots * a.m, 64);
    p.group_slots = p.groups > 1 ? worker_slots : p.slots;
    // D of bfloat16 operands, 16 bits of it: by one term, as many bits as the results have, they would be off by 1.4 times their own rounding, and by up to twice it
    // where they hang on one entry of D.
    p.prob_terms = p.x_terms > 1 || p.w_terms > 1 ? 3 : 2;
    p.pitch = up(a.cols, 8);
    p.parts_pitch = up(a.cols, 4);
    const int64_t per_word = p.w_packed ? p.groups * p.w_terms * p.pitch * 2 : 0, per_prob = gradient ? p.slots * p.prob_terms * 2 : 0;
    int64_t most = up(a.vocab, 256);
    if (per_word && kWeightBytes / per_word < most) most = kWeightBytes / per_word / 256 * 256;
    if (per_prob && kPieceBytes / per_prob < most) most = kPieceBytes / per_prob / 256 * 256;
    if (most < kMinPiece) most = kMinPiece;
    p.pieces = (int)((a.vocab + most - 1) / most);
    p.piece = up((a.vocab + p.pieces - 1) / p.pieces, 256);
    // with few tiles of rows, pieces of as many tiles as make whole rounds (2 x 132 tokens, half of them masked, 40576 words by 5568 columns in binary32: 1,040 us, by
    // pieces of any length 1,120; the gradient 2,160 and 2,235)
    p.sum_blocks = p.group_slots <= 128 ? 1 : 2;
    const int64_t row_tiles = up(p.group_slots, p.sum_blocks * 128) / (p.sum_blocks * 128) * p.groups, units = 2 * kHeadPairs / p.sum_blocks, round = units / row_tiles * 256;
    if (p.pieces > 1 && round > 0 && round <= most) p.piece = most / round * round;
    p.pieces = (int)((a.vocab + p.piece - 1) / p.piece);
    // a tile of 128 columns where there are fewer of 256 than there are SMs, or pairs, for them
    const int64_t sum_tiles = row_tiles * (p.piece / 256);
    p.sum_cols = sum_tiles < units ? 128 : 256;
    // Few tiles of a long contraction: it is cut, the parts' logits are kept and joined by the kernel that needs them.  In one part a tile's stages follow one
    // another on one SM or pair however idle the others are.
    HeadTcArgs pairs = {};
    set_pairs(&pairs, p.x_terms, p.w_terms);
    const int64_t blocks_of_64 = (a.cols + 63) / 64, stages = blocks_of_64 * pairs.pairs;
    int64_t logits_parts = units / sum_tiles;
    if (logits_parts > stages / 8) logits_parts = stages / 8;
    if (logits_parts > blocks_of_64) logits_parts = blocks_of_64;
    // (A stage takes about a quarter of a microsecond, the parts' way through memory and the other kernel as much as some forty.)
    p.logits_parts = p.pieces == 1 && logits_parts > 1 && stages - stages / logits_parts >= 40 ? (int)logits_parts : 0;
    p.logits_pitch = up(a.vocab, 4);
    p.tile_cols = a.cols <= 128 ? 128 : 256;                          // of the gradients: few tiles of dx are cut along the words instead
    p.most_splits = (int)(p.piece / 64 / 8);                          // parts of eight stages and more
    if (p.most_splits < 1) p.most_splits = 1;
    p.sum_words = head_part_words(p.sum_cols, p.x_terms, p.w_terms, a.cols);
    p.part_pitch = up(a.vocab, 256) / p.sum_words;
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
    p.part = take(p.logits_parts ? p.logits_parts * p.slots * p.logits_pitch * 4 : gradient ? 0 : p.slots * p.part_pitch * 8);
    p.probs = take(p.piece * per_prob);
    p.parts = take(gradient && a.dx.data ? p.slots * p.parts_pitch * 4 : 0);
    p.extra = take(gradient && a.dx.data ? (int64_t)kHeadPairs * kHeadRows * p.tile_cols * 4 : 0);
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
    float most = 0.f;
    bool number = true;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = fmaxf(most, fabsf(f[k])), number = number && f[k] == f[k];
    const bool plain = number && most <= 3.3895314e38f;                // bfloat16's largest: nothing rounds to infinity
#pragma unroll
    for (int t = 0; t < TERMS; ++t) {
        uint32_t v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (!plain) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float &e = f[2 * k + i];
                    __nv_bfloat16 h = __float2bfloat16_rn(e);
                    // (a finite number may round to infinity: then the term is the largest finite one)
                    if (fabsf(e) < INFINITY && !(fabsf(__bfloat162float(h)) < INFINITY)) h = __ushort_as_bfloat16(e < 0.f ? 0xff7f : 0x7f7f);
                    e = fabsf(e) < INFINITY ? e - __bfloat162float(h) : 0.f;
                    v[k] = i ? v[k] | (uint32_t)__bfloat16_as_ushort(h) << 16 : __bfloat16_as_ushort(h);
                }
                continue;
            }
            v[k] = two_bf16(f[2 * k], f[2 * k + 1]);
            if (t + 1 < TERMS) {
                f[2 * k] -= __uint_as_float(v[k] << 16);
                f[2 * k + 1] -= __uint_as_float(v[k] & 0xffff0000u);
            }
        }
        *reinterpret_cast<uint4 *>(to + t * plane) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

// Eight entries of a row on their way: as they lie (VECTORS), or as the aligned words around them, of those that hold an entry of the row.
template <typename T>
struct Eight {
    static constexpr int kLoads = 8 * sizeof(T) / 16;
    uint4 q[kLoads + 1];
    __device__ __forceinline__ void load(const T *row, int64_t c, int64_t cols, bool vectors) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(row + c), end = reinterpret_cast<uintptr_t>(row + cols);
        const uint4 *words = reinterpret_cast<const uint4 *>(at & ~(uintptr_t)15);
#pragma unroll
        for (int k = 0; k < kLoads + 1; ++k) {
            q[k] = make_uint4(0, 0, 0, 0);
            if (row && c < cols && (k < kLoads || !vectors) && reinterpret_cast<uintptr_t>(words + k) < end) q[k] = words[k];
        }
    }
    // of bfloat16: as they are, zeros behind the row's end
    __device__ __forceinline__ uint4 bits(const T *row, int64_t c, int64_t cols, bool vectors) const {
        uint4 v = vectors ? q[0] : shifted<2>(q[0], q[1], (unsigned)(reinterpret_cast<uintptr_t>(row + c) & 15));
        if (!row || c + 8 > cols) {
            const int left = row && c < cols ? (int)(cols - c) : 0;
            auto keep = [&](uint32_t w, int at) { return left >= at + 2 ? w : left == at + 1 ? w & 0xffffu : 0u; };
            v = make_uint4(keep(v.x, 0), keep(v.y, 2), keep(v.z, 4), keep(v.w, 6));
        }
        return v;
    }
    // of binary32
    __device__ __forceinline__ void get(float (&f)[8], const T *row, int64_t c, int64_t cols, bool vectors) const {
        const unsigned off = vectors ? 0u : (unsigned)(reinterpret_cast<uintptr_t>(row + c) & 15);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const uint4 v = vectors ? q[k] : shifted<sizeof(T)>(q[k], q[k + 1], off);
            f[4 * k] = __uint_as_float(v.x), f[4 * k + 1] = __uint_as_float(v.y), f[4 * k + 2] = __uint_as_float(v.z), f[4 * k + 3] = __uint_as_float(v.w);
        }
        if (!row || c + 8 > cols)
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = row && c + i < cols ? f[i] : 0.f;
    }
};

// Some threads rewrite a row of cols entries (NULL: zeros), eight to a thread and turn.
template <typename T, int TERMS>
__device__ __forceinline__ void row_terms(const T *from, __nv_bfloat16 *to, int64_t cols, int64_t pitch, int64_t plane, bool vectors, int thread, int threads) {
    for (int64_t c = thread * 8; c < pitch; c += threads * 8) {
        Eight<T> e;
        e.load(from, c, cols, vectors);
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4 *>(to + c) = e.bits(from, c, cols, vectors);
        } else {
            float f[8];
            e.get(f, from, c, cols, vectors);
            put_terms<TERMS>(f, to + c, plane);
        }
    }
}

// Threads for a row: a power of two, a warp at least and a block at most.
int threads_log2(int64_t pitch) {
    int log2 = 5;
    while (log2 < 8 && (8 << log2) < pitch) ++log2;
    return log2;
}

struct SlotsArgs {
    HeadArgs a;
    Plan p;
    int vectors, threads_log2;
};

template <typename V>
__host__ __device__ __forceinline__ V *at(const HeadArgs &a, int64_t offset) {
    return reinterpret_cast<V *>(static_cast<uint8_t *>(a.workspace) + offset);
}

// blockIdx.y is the worker.  ALONE: of a few tokens every block finds the order itself, which saves a launch (and 2 us of 25 for 1648 tokens, 449 words by 300
// columns), but reads all workers' tokens before its own (8 x 1000 tokens, 200 words by 64 columns: 26 us, by the other kernel 24; 500 x 1 44, 19; 8000 x 1 2,290, 70).
constexpr int64_t kAloneTokens = 2048;
constexpr int kAloneWorkers = 32;

template <typename T, int TERMS, bool ALONE>
__global__ void __launch_bounds__(256) head_slots_kernel(const SlotsArgs args) {
    __shared__ int scratch[8];
    __shared__ short order[ALONE ? kAloneTokens : 1];
    const HeadArgs &a = args.a;
    const Plan &p = args.p;
    pdl_wait();
    pdl_launch_dependents();
    const int worker = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int *counts = at<int>(a, p.counts);
    auto given = [&](int64_t row) { return (uint32_t)a.targets[row] < (uint64_t)a.vocab; };
    int count = 0;
    if constexpr (ALONE) {
        for (int t0 = 0; t0 < (int)a.n; t0 += 256) {
            const int t = t0 + threadIdx.x;
            const bool mine = t < a.n && given(worker * a.n + t);
            const unsigned votes = __ballot_sync(0xffffffffu, mine);
            if (lane == 0) scratch[warp] = __popc(votes);
            __syncthreads();
            int before = count;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                if (w < warp) before += scratch[w];
                count += scratch[w];
            }
            const int k = before + __popc(votes & ((1u << lane) - 1));
            if (mine) order[k] = (short)t;
            if (blockIdx.x == 0 && t < a.n) at<int>(a, p.rank)[worker * a.n + t] = mine ? k : -1;
            __syncthreads();
        }
    } else {
        count = counts[worker];
    }
    const int lot = p.lot, filled = (count + lot - 1) / lot * lot;
    int begin = 0;
    if (p.groups > 1) {
        begin = (int)(worker * p.group_slots);
    } else {                                                          // behind the workers before
        if constexpr (ALONE) {
            for (int i = warp; i < worker; i += 8) {
                int others = 0;
#pragma unroll 4
                for (int t = lane; t < (int)a.n; t += 32) others += given(i * a.n + t);
                others = __reduce_add_sync(0xffffffffu, others);
                if (lane == 0) begin += (others + lot - 1) / lot * lot;
            }
        } else {
            for (int i = threadIdx.x; i < worker; i += 256) begin += (counts[i] + lot - 1) / lot * lot;
        }
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
    const int threads = 1 << args.threads_log2, thread = threadIdx.x & (threads - 1), rows_of_block = 256 >> args.threads_log2;
    for (int k = blockIdx.x * rows_of_block + (threadIdx.x >> args.threads_log2); k < filled; k += gridDim.x * rows_of_block) {
        const int token = k >= count ? -1 : ALONE ? order[k] : at<int>(a, p.list)[worker * a.n + k];
        const int64_t slot = begin + k, row = worker * a.n + token;
        if (thread == 0) {
            at<int>(a, p.target)[slot] = token >= 0 ? a.targets[row] : -1;
            if (a.g) {
                at<float>(a, p.lse)[slot] = token >= 0 ? a.lse_in[row] : -INFINITY;
                at<float>(a, p.g)[slot] = token >= 0 ? a.g[row] * a.scale : 0.f;
            }
        }
        const T *from = token >= 0 ? static_cast<const T *>(a.x.data) + worker * a.x.group + token * a.x.row : nullptr;
        row_terms<T, TERMS>(from, at<__nv_bfloat16>(a, p.x) + slot * p.pitch, a.cols, p.pitch, p.slots * p.pitch, args.vectors, thread, threads);
    }
}

// Words v0 .. v0 + words - 1 of every group's weights: [group][term][piece][pitch].  The first piece's are rewritten beside the tokens' kernels, which
// touch none of them and started behind all that came before this call; the end is waited for all the same, for the sake of the kernel that comes next.
template <typename T, int TERMS>
__global__ void __launch_bounds__(256) head_words_kernel(const T *w, int64_t ldw, int64_t cols, int64_t pitch, int64_t v0, int words, int64_t piece, int64_t total,
                                                         __nv_bfloat16 *out, int vectors, int threads_log2, int beside) {
    if (!beside) pdl_wait();
    pdl_launch_dependents();
    const int threads = 1 << threads_log2, rows_of_block = 256 >> threads_log2;
    for (int64_t q = (int64_t)blockIdx.x * rows_of_block + (threadIdx.x >> threads_log2); q < total; q += (int64_t)gridDim.x * rows_of_block) {
        const uint32_t group = (uint32_t)q / (uint32_t)words, v = (uint32_t)q - group * words;
        row_terms<T, TERMS>(w + group * ldw + (v0 + v) * cols, out + ((int64_t)group * TERMS * piece + v) * pitch, cols, pitch, piece * pitch, vectors, threadIdx.x & (threads - 1), threads);
    }
    if (beside) pdl_wait();
}

// ---- few tokens

// Log-sum-exp in parts: the largest so far and the sum of exponentials beside it.
__device__ __forceinline__ void add_part(float2 &to, float top, float sum) {
    const float most = fmaxf(to.x, top), beside = most == -INFINITY ? 0.f : most;
    to.y = to.y * expf(to.x - beside) + sum * expf(top - beside);          // exp(-inf) of a part that has nothing yet; NaN stays in the sums
    to.x = most;
}

// Every warp takes WORDS words at a time, its lanes eight columns of 256 (neighbours where all rows are aligned, else every 32nd), and asks for the next
// AHEAD times 256 columns before it multiplies the last ones; hidden states are kept in shared memory in binary32.  Bound by the weights' way from memory.
template <typename T, typename P, int R, bool VECTORS>
__global__ void __launch_bounds__(256, 2) head_few_kernel(const HeadArgs a, const Plan p) {
    constexpr int WORDS = 2, AHEAD = VECTORS && sizeof(P) == 2 && R <= 2 ? 4 : 2, kRegs = VECTORS ? (int)sizeof(P) * 2 : 8;
    extern __shared__ __align__(16) float held[];            // [row][column]; of eight neighbours the latter four in a second half (VECTORS)
    __shared__ float2 of_warp[8][R];
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // neighbouring blocks take the same words with R tokens each, so that all but one find the words in L2
    const int64_t of_group = p.groups > 1 ? a.n : a.m * a.n;
    const int lots = (int)((of_group + R - 1) / R), block = blockIdx.x / lots, lot = blockIdx.x - block * lots, blocks = gridDim.x / lots;
    const int64_t row0 = blockIdx.y * of_group + lot * R;
    const int group_rows = (int)min((int64_t)R, of_group - lot * R);
    const int cols = (int)a.cols, padded = (cols + 256 * AHEAD - 1) / (256 * AHEAD) * (256 * AHEAD);
    const P *w = static_cast<const P *>(a.w) + blockIdx.y * a.ldw;
    const int64_t step = (int64_t)blocks * 8 * WORDS;
    uint32_t next[AHEAD][WORDS][kRegs];
    auto ask = [&](int64_t v0, int c0) {
#pragma unroll
        for (int h = 0; h < AHEAD; ++h)
#pragma unroll
            for (int k = 0; k < WORDS; ++k) {
                const P *from = w + (v0 + k) * cols + c0 + h * 256;
                const int left = v0 + k < a.vocab ? cols - c0 - h * 256 : 0;
                if constexpr (VECTORS) {
#pragma unroll
                    for (int i = 0; i < kRegs / 4; ++i) {
                        const uint4 q = lane * 8 < left ? __ldcs(reinterpret_cast<const uint4 *>(from + lane * 8) + i) : make_uint4(0, 0, 0, 0);
                        next[h][k][4 * i] = q.x, next[h][k][4 * i + 1] = q.y, next[h][k][4 * i + 2] = q.z, next[h][k][4 * i + 3] = q.w;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) next[h][k][i] = lane + 32 * i < left ? __float_as_uint(value_of(from + lane + 32 * i)) : 0u;
                }
            }
    };
    int64_t v0 = ((int64_t)block * 8 + warp) * WORDS;
    ask(v0, 0);
    int target = -1;                                         // of the lane's row
    if (lane < group_rows) target = a.targets[row0 + lane];
    if ((uint32_t)target >= (uint64_t)a.vocab) target = -1;
    const unsigned given = __ballot_sync(0xffffffffu, target >= 0);
    for (int r = 0; r < R; ++r)
        for (int c = threadIdx.x; c < padded; c += 256) {
            float v = 0.f;
            if (c < cols && (given >> r & 1)) {
                const int64_t row = row0 + r, worker = row / a.n;
                v = value_of(static_cast<const T *>(a.x.data) + worker * a.x.group + (row - worker * a.n) * a.x.row + c);
            }
            held[r * padded + (VECTORS ? (c & 4 ? padded / 2 : 0) + (c >> 3) * 4 + (c & 3) : c)] = v;
        }
    __syncthreads();
    float2 mine = make_float2(-INFINITY, 0.f);               // of the lane's row
    while (v0 < a.vocab) {
        Two sum[2][WORDS][R] = {};                           // two chains of additions each
        const int64_t following = v0 + step;
        for (int c0 = 0; c0 < padded; c0 += 256 * AHEAD) {
            uint32_t now[AHEAD][WORDS][kRegs];
#pragma unroll
            for (int h = 0; h < AHEAD; ++h)
#pragma unroll
                for (int k = 0; k < WORDS; ++k)
#pragma unroll
                    for (int i = 0; i < kRegs; ++i) now[h][k][i] = next[h][k][i];
            const bool same = c0 + 256 * AHEAD < padded;
            ask(same ? v0 : following, same ? c0 + 256 * AHEAD : 0);
#pragma unroll
            for (int h = 0; h < AHEAD; ++h) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float *x = held + r * padded;
                    const int c = c0 + h * 256;
                    float f[8];
                    if constexpr (VECTORS) {
                        const float4 lo = *reinterpret_cast<const float4 *>(x + (c >> 1) + lane * 4), hi = *reinterpret_cast<const float4 *>(x + padded / 2 + (c >> 1) + lane * 4);
                        f[0] = lo.x, f[1] = lo.y, f[2] = lo.z, f[3] = lo.w, f[4] = hi.x, f[5] = hi.y, f[6] = hi.z, f[7] = hi.w;
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[i] = x[c + lane + 32 * i];
                    }
#pragma unroll
                    for (int k = 0; k < WORDS; ++k)
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            const uint32_t *q = now[h][k];
                            const Two e = kRegs == 8 ? Two{__uint_as_float(q[i % kRegs]), __uint_as_float(q[(i + 1) % kRegs])}
                                                     : Two{__uint_as_float(q[i / 2] << 16), __uint_as_float(q[i / 2] & 0xffff0000u)};
                            Two &to = sum[h & 1][k][r];
                            to = fma2(e, Two{f[i], f[i + 1]}, to);
                        }
                }
            }
        }
        const int words = (int)min((int64_t)WORDS, a.vocab - v0);
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            float z = 0.f;                                   // of the lane's row
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float s = warp_sum((sum[0][k][r].x + sum[0][k][r].y) + (sum[1][k][r].x + sum[1][k][r].y));
                if (lane == r) z = s;
            }
            z *= a.scale;
            if (lane < group_rows && k < words) {
                if (v0 + k == target) at<float>(a, p.target_logit)[row0 + lane] = z;
                add_part(mine, z, 1.f);
            }
        }
        v0 = following;
    }
    if (lane < R) of_warp[warp][lane] = mine;
    __syncthreads();
    if ((int)threadIdx.x < group_rows) {
        mine = of_warp[0][threadIdx.x];
        for (int k = 1; k < 8; ++k) add_part(mine, of_warp[k][threadIdx.x].x, of_warp[k][threadIdx.x].y);
        at<float2>(a, p.part)[(row0 + threadIdx.x) * p.part_pitch + block] = mine;
    }
}

// ---- ends (a call's last kernel lets nothing start before its end)

// lse and log probability of every token from its parts of the vocabulary: a warp per token.
__global__ void __launch_bounds__(256) head_join_kernel(const HeadArgs a, const Plan p, int parts) {
    pdl_wait();
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    if (row >= a.m * a.n) return;
    const int rank = p.few ? ((uint32_t)a.targets[row] < (uint64_t)a.vocab ? 0 : -1) : at<int>(a, p.rank)[row];
    float lse = 0.f, logprob = 0.f;
    if (rank >= 0) {
        const int64_t slot = p.few ? row : at<int>(a, p.begin)[row / a.n] + rank;
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

// The sums of four neighbouring words' parts.
__device__ __forceinline__ float4 four_logits(const float *parts, int count, int64_t plane) {
    float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = 0; i < count; ++i) {
        const float4 v = *reinterpret_cast<const float4 *>(parts + i * plane);
        z.x += v.x, z.y += v.y, z.z += v.z, z.w += v.w;
    }
    return z;
}

// lse and log probability of every token from its logits in parts: a block per token.
__global__ void __launch_bounds__(256) head_logits_kernel(const HeadArgs a, const Plan p) {
    __shared__ float2 of_warp[8];
    __shared__ float target_logit;
    pdl_wait();
    const int64_t row = blockIdx.x;
    const int rank = at<int>(a, p.rank)[row], lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (rank < 0) {
        if (threadIdx.x == 0 && a.lse) a.lse[row] = 0.f;
        if (threadIdx.x == 0 && a.logprobs) a.logprobs[row] = 0.f;
        return;
    }
    const int64_t slot = at<int>(a, p.begin)[row / a.n] + rank, plane = p.slots * p.logits_pitch;
    const float *logits = at<float>(a, p.part) + slot * p.logits_pitch;
    const int target = a.targets[row];
    float2 mine = make_float2(-INFINITY, 0.f);
    for (int v0 = threadIdx.x * 4; v0 < (int)a.vocab; v0 += 1024) {
        const float4 four = four_logits(logits + v0, p.logits_parts, plane);
        float z[4] = {four.x * a.scale, four.y * a.scale, four.z * a.scale, four.w * a.scale};
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (v0 + k == target) target_logit = z[k];
            if (v0 + k >= (int)a.vocab) z[k] = -INFINITY;
            top = fmaxf(top, z[k]);
        }
        const float beside = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += expf(z[k] - beside);
        add_part(mine, top, sum);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float top = __shfl_xor_sync(0xffffffffu, mine.x, d), sum = __shfl_xor_sync(0xffffffffu, mine.y, d);
        add_part(mine, top, sum);
    }
    if (lane == 0) of_warp[warp] = mine;
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < 8; ++w) add_part(mine, of_warp[w].x, of_warp[w].y);
    const double beside = mine.x == -INFINITY ? 0. : mine.x, log_sum = log((double)mine.y);
    if (a.lse) a.lse[row] = (float)(beside + log_sum);
    if (a.logprobs) a.logprobs[row] = mine.y == 0.f ? -INFINITY : (float)((double)target_logit - beside - log_sum);
}

// D from logits in parts, eight words of a slot a thread: blockIdx.y is the group.
template <int TERMS>
__global__ void __launch_bounds__(256) head_probs_kernel(const HeadArgs a, const Plan p) {
    pdl_wait();
    pdl_launch_dependents();
    const int begin = p.groups > 1 ? at<int>(a, p.begin)[blockIdx.y] : 0, end = p.groups > 1 ? at<int>(a, p.end)[blockIdx.y] : at<int>(a, p.total)[1];
    const int64_t per_row = p.piece / 8, total = (end - begin) * per_row, plane = p.slots * p.logits_pitch;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
        const int64_t slot = begin + q / per_row, v0 = q % per_row * 8;
        const float lse = at<float>(a, p.lse)[slot], g = at<float>(a, p.g)[slot];
        const int target = at<int>(a, p.target)[slot];
        const float *logits = at<float>(a, p.part) + slot * p.logits_pitch + v0;
        float f[8] = {};
        if (lse != -INFINITY)                              // else no token, or nothing but logits of minus infinity
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (v0 + 4 * h >= a.vocab) break;
                const float4 four = four_logits(logits + 4 * h, p.logits_parts, plane);
                const float z[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int64_t v = v0 + 4 * h + k;
                    f[4 * h + k] = v < a.vocab ? (expf(fmaf(z[k], a.scale, -lse)) - (v == target ? 1.f : 0.f)) * -g : 0.f;
                }
            }
        put_terms<TERMS>(f, at<__nv_bfloat16>(a, p.probs) + slot * p.piece + v0, p.slots * p.piece);
    }
}

// dx, four neighbouring entries a thread, rounded once; zero without a target.  Tiles that were cut have further parts.
template <typename T>
__global__ void __launch_bounds__(256) head_inputs_kernel(const HeadArgs a, const Plan p, uint32_t pairs, int vectors) {
    pdl_wait();
    const int64_t per_row = p.parts_pitch / 4, total = (int64_t)a.m * a.n * per_row;
    const uint32_t bound = (uint32_t)((p.group_slots + kHeadRows - 1) / kHeadRows), used = (uint32_t)((at<int>(a, p.total)[1] + kHeadRows - 1) / kHeadRows);
    const uint32_t row_tiles = p.groups > 1 ? bound : min(bound, used), col_tiles = (uint32_t)((a.cols + p.tile_cols - 1) / p.tile_cols);
    const uint32_t tiles = row_tiles * col_tiles * p.groups, whole = tiles / pairs * pairs;
    const int splits = head_splits(tiles, pairs, p.most_splits);
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
        const int64_t row = q / per_row, c = (q - row * per_row) * 4, worker = row / a.n;
        const int rank = at<int>(a, p.rank)[row];
        float s[4] = {};
        if (rank >= 0) {
            const int slot = at<int>(a, p.begin)[worker] + rank;
            const float4 v = *reinterpret_cast<const float4 *>(at<float>(a, p.parts) + slot * p.parts_pitch + c);
            s[0] = v.x, s[1] = v.y, s[2] = v.z, s[3] = v.w;
            const int in_group = p.groups > 1 ? rank : slot, col = (int)(c / p.tile_cols);
            const uint32_t tile = (p.groups > 1 ? (uint32_t)worker * row_tiles * col_tiles : 0) + head_tile_number(in_group / kHeadRows, col, row_tiles, col_tiles);
            if (tile >= whole)
                for (int i = 1; i < splits; ++i) {
                    const int64_t item = (int64_t)(tile - whole) * splits + i;
                    const float4 u = *reinterpret_cast<const float4 *>(at<float>(a, p.extra) + (item * kHeadRows + in_group % kHeadRows) * p.tile_cols + (c - col * p.tile_cols));
                    s[0] += u.x, s[1] += u.y, s[2] += u.z, s[3] += u.w;
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


cudaError_t fill_slots(int type, const HeadArgs &a, const Plan &p, cudaStream_t s) {
    const bool alone = a.m <= kAloneWorkers && a.m * a.n <= kAloneTokens;
    if (!alone) {
        const cudaError_t e = launch_chained(head_order_kernel, dim3(a.m), dim3(kOrderThreads), 0, s, true, a.targets, a.n, a.vocab, at<int>(a, p.counts), at<int>(a, p.list), at<int>(a, p.rank));
        if (e != cudaSuccess) return e;
    }
    const int elem = type == ZENO_F32 ? 4 : 2;
    const SlotsArgs args = {a, p, a.cols % 8 == 0 && aligned_to(a.x, a.m, a.n, elem, 16), threads_log2(p.pitch)};
    const int64_t rows_of_block = 256 >> args.threads_log2, blocks = (up(a.n, p.lot) + rows_of_block - 1) / rows_of_block;
    const dim3 grid((unsigned)(blocks < 2048 ? blocks : 2048), a.m);
    auto *kernel = type == ZENO_F32 ? (alone ? head_slots_kernel<float, 3, true> : head_slots_kernel<float, 3, false>)
                                    : (alone ? head_slots_kernel<__nv_bfloat16, 1, true> : head_slots_kernel<__nv_bfloat16, 1, false>);
    return launch_chained(kernel, grid, dim3(256), 0, s, true, args);
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
    const int log2 = threads_log2(p.pitch), rows_of_block = 256 >> log2;
    const dim3 grid = grid_for((total + rows_of_block - 1) / rows_of_block);
    return param_type == ZENO_F32 ? launch_chained(head_words_kernel<float, 3>, grid, dim3(256), 0, s, true, static_cast<const float *>(a.w), a.ldw, a.cols, p.pitch, v0,
                                                   (int)words, p.piece, total, out, vectors, log2, (int)(v0 == 0))
                                  : launch_chained(head_words_kernel<__nv_bfloat16, 1>, grid, dim3(256), 0, s, true, static_cast<const __nv_bfloat16 *>(a.w), a.ldw, a.cols,
                                                   p.pitch, v0, (int)words, p.piece, total, out, vectors, log2, (int)(v0 == 0));
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
    h.tile_cols = p.sum_cols;
    h.blocks = p.sum_blocks;
    return h;
}

// Logits in parts.
cudaError_t launch_logits(HeadTcArgs h, const HeadArgs &a, const Plan &p, cudaStream_t s) {
    h.step = HeadStep::kLogits;
    h.tile_cols = 256;
    h.logits = at<float>(a, p.part);
    h.logits_pitch = p.logits_pitch;
    h.logits_parts = p.logits_parts;
    h.bf16_result = 0;
    return launch_head_tc(h, s);
}

Operand slots_operand(const HeadArgs &a, const Plan &p) { return Operand{at<void>(a, p.x), a.cols, p.slots, p.pitch, p.slots * p.pitch, p.x_terms}; }

template <typename T, typename P, int R, bool VECTORS>
cudaError_t few(const HeadArgs &a, const Plan &p, int64_t rows, cudaStream_t s) {
    auto *kernel = head_few_kernel<T, P, R, VECTORS>;
    static PerDeviceOnce once;
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess && once.need(device)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, R * (int)kFewCols * 4);
        if (e == cudaSuccess) once.mark(device);
    }
    return e == cudaSuccess ? launch_chained(kernel, dim3((unsigned)(p.few_blocks * ((rows + R - 1) / R)), p.groups), dim3(256), (size_t)(R * up(a.cols, 1024) * 4), s, true, a, p) : e;
}

template <typename T, typename P>
cudaError_t few_rows(const HeadArgs &a, const Plan &p, cudaStream_t s) {
    const int64_t rows = p.groups > 1 ? a.n : a.m * a.n;
    const bool vectors = a.cols % 8 == 0 && reinterpret_cast<uintptr_t>(a.w) % 16 == 0 && (p.groups == 1 || a.ldw * sizeof(P) % 16 == 0);
    if (rows <= 1) return vectors ? few<T, P, 1, true>(a, p, rows, s) : few<T, P, 1, false>(a, p, rows, s);
    if (rows <= 2) return vectors ? few<T, P, 2, true>(a, p, rows, s) : few<T, P, 2, false>(a, p, rows, s);
    return vectors ? few<T, P, kFew, true>(a, p, rows, s) : few<T, P, kFew, false>(a, p, rows, s);
}

}  // namespace

int64_t head_workspace(int type, int param_type, bool gradient, const HeadArgs &a) { return a.m > 0 && a.n > 0 ? plan_head(type, param_type, gradient, a).bytes : 0; }

cudaError_t launch_head_logprobs(int type, int param_type, const HeadArgs &a, cudaStream_t s) {
    const Plan p = plan_head(type, param_type, false, a);
    if (p.few) {
        const cudaError_t e = type == ZENO_F32 ? (param_type == ZENO_F32 ? few_rows<float, float>(a, p, s) : few_rows<float, __nv_bfloat16>(a, p, s))
                                               : (param_type == ZENO_F32 ? few_rows<__nv_bfloat16, float>(a, p, s) : few_rows<__nv_bfloat16, __nv_bfloat16>(a, p, s));
        if (e != cudaSuccess) return e;
        return launch_chained(head_join_kernel, dim3((unsigned)((a.m * a.n + 7) / 8)), dim3(256), 0, s, true, a, p, p.few_blocks);
    }
    cudaError_t e = fill_slots(type, a, p, s);
    for (int i = 0; i < p.pieces && e == cudaSuccess; ++i) {
        HeadTcArgs h = common(a, p, HeadStep::kSums);
        h.v0 = i * p.piece;
        h.piece = a.vocab - h.v0 < p.piece ? a.vocab - h.v0 : p.piece;
        e = piece_weights(param_type, a, p, h.v0, h.piece, &h.b, &h.b_row0, s);
        if (e != cudaSuccess) break;
        h.a = slots_operand(a, p);
        set_pairs(&h, p.x_terms, p.w_terms);
        if (p.logits_parts) {
            e = launch_logits(h, a, p, s);
            return e == cudaSuccess ? launch_chained(head_logits_kernel, dim3((unsigned)(a.m * a.n)), dim3(256), 0, s, true, a, p) : e;
        }
        h.part = at<float2>(a, p.part);
        h.part_pitch = p.part_pitch;
        h.target_logit = at<float>(a, p.target_logit);
        e = launch_head_tc(h, s);
    }
    if (e != cudaSuccess) return e;
    return launch_chained(head_join_kernel, dim3((unsigned)((a.m * a.n + 7) / 8)), dim3(256), 0, s, true, a, p, (int)(up(a.vocab, p.sum_words) / p.sum_words));
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
        if (p.logits_parts) {
            e = launch_logits(h, a, p, s);
            if (e != cudaSuccess) break;
            const int64_t blocks = (p.group_slots * (p.piece / 8) + 255) / 256;
            const dim3 grid((unsigned)(blocks < 148 * 8 ? blocks : 148 * 8), p.groups);
            e = launch_chained(p.prob_terms == 2 ? head_probs_kernel<2> : head_probs_kernel<3>, grid, dim3(256), 0, s, true, a, p);
        } else {
            e = launch_head_tc(h, s);
        }
        if (e != cudaSuccess) break;
        const Operand probs = {h.probs, h.piece, p.slots, p.piece, p.slots * p.piece, p.prob_terms};
        if (a.dx.data) {
            h.step = HeadStep::kInputs;
            h.bf16_result = type == ZENO_BF16;
            h.a = probs;
            set_pairs(&h, p.prob_terms, p.w_terms);
            h.parts = at<float>(a, p.parts);
            h.parts_pitch = p.parts_pitch;
            h.extra = at<float>(a, p.extra);
            h.most_splits = p.most_splits;
            h.tile_cols = p.tile_cols;
            h.blocks = 2;
            h.accumulate = i > 0;
            e = launch_head_tc(h, s);
            if (e != cudaSuccess) break;
        }
        if (a.dw) {
            h.step = HeadStep::kWeights;
            h.bf16_result = param_type == ZENO_BF16;
            h.tile_cols = p.tile_cols;
            h.blocks = 2;
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
    const uint32_t pairs = head_pairs();
    return type == ZENO_F32 ? launch_chained(head_inputs_kernel<float>, grid_for(blocks), dim3(256), 0, s, true, a, p, pairs, vectors)
                            : launch_chained(head_inputs_kernel<__nv_bfloat16>, grid_for(blocks), dim3(256), 0, s, true, a, p, pairs, vectors);
}

}  // namespace zeno

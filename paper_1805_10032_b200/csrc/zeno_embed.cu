// A language model's embedding, y_t = scale E[id_t], and its gradient for every worker, dE[v] = scale sum over the tokens with id v of dy_t.
//
// Forward: a lane gathers 16 bytes at a time, two of four rows in flight; bound by memory.
// Backward: every row of the table is written once, mostly zeros, and no row is summed by atomics.  A first kernel sorts each worker's token positions by
// id: a block per class of ids counts what each of its warps finds in a stretch of the tokens, and places the positions, rows in order, positions
// in order within a row.  The second one writes the rows without tokens, then walks over the sorted positions, a warp to 32 of them and 512 bytes of
// their rows, whichever rows of the table they belong to: frequent ids cost no more than others.  A row of up to 32 positions is summed by the warp in whose stretch it
// begins; what the warps have of a longer one is left for the third kernel, which adds these parts in their order.
#include "zeno_operators.h"

namespace zeno {

namespace {

// N entries as they lie in memory, in words (a single bfloat16 in half of one): arrays of bfloat16 would go to local memory.
template <typename T, int N>
struct Pack {
    static constexpr int kWords = sizeof(T) * N < 4 ? 1 : (int)sizeof(T) * N / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T *from) {
        if constexpr (sizeof(T) * N == 2) w[0] = *reinterpret_cast<const unsigned short *>(from);
        else if constexpr (sizeof(T) * N == 4) w[0] = *reinterpret_cast<const uint32_t *>(from);
        else if constexpr (sizeof(T) * N == 8) reinterpret_cast<uint2 &>(w) = *reinterpret_cast<const uint2 *>(from);
        else
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 q = *reinterpret_cast<const uint4 *>(from + i * (int)(4 / sizeof(T)));
                w[i] = q.x, w[i + 1] = q.y, w[i + 2] = q.z, w[i + 3] = q.w;
            }
    }
    __device__ __forceinline__ void store(T *to) const {
        if constexpr (sizeof(T) * N == 2) *reinterpret_cast<unsigned short *>(to) = (unsigned short)w[0];
        else if constexpr (sizeof(T) * N == 4) *reinterpret_cast<uint32_t *>(to) = w[0];
        else if constexpr (sizeof(T) * N == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
        else
#pragma unroll
            for (int i = 0; i < kWords; i += 4) *reinterpret_cast<uint4 *>(to + i * (int)(4 / sizeof(T))) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void set(int i, float v) {
        if constexpr (sizeof(T) == 4) {
            w[i] = __float_as_uint(v);
        } else {
            const uint32_t h = __bfloat16_as_ushort(__float2bfloat16_rn(v));
            w[i / 2] = i & 1 ? w[i / 2] | h << 16 : h;              // the lower half first
        }
    }
};

// 2^lanes_log2 lanes to a row, kRows rows and kPieces pieces of each in flight; blockIdx.y: which pieces of the rows.
template <typename T, typename P, int N>
__global__ void __launch_bounds__(256, 4) embed_kernel(const EmbedArgs a, int per_row, int rows, int lanes_log2) {
    constexpr int kRows = 4, kPieces = 2;
    pdl_wait();
    const int lane = threadIdx.x & 31, l = lane & ((1 << lanes_log2) - 1), sub = lane >> lanes_log2, at_once = 32 >> lanes_log2;
    const int64_t row0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * kRows * at_once + sub;
    const int piece0 = blockIdx.y * (kPieces << lanes_log2) + l;
    int id[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) id[r] = row0 + r * at_once < rows ? a.tokens[row0 + r * at_once] : -1;
    Pack<P, N> in[kRows][kPieces];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const bool given = (uint32_t)id[r] < (uint64_t)a.vocab;
        const P *from = static_cast<const P *>(a.table) + (given ? (a.ldt ? (uint32_t)(row0 + r * at_once) / (uint32_t)a.n * a.ldt : 0) + id[r] * a.cols : 0);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int piece = piece0 + (k << lanes_log2);
            in[r][k] = Pack<P, N>{};
            if (given && piece < per_row) in[r][k].load(from + (int64_t)piece * N);
        }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int64_t row = row0 + r * at_once;
        if (row >= rows) break;
        T *to = static_cast<T *>(a.y.data) + a.y.at(row);
        const bool given = (uint32_t)id[r] < (uint64_t)a.vocab;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int piece = piece0 + (k << lanes_log2);
            Pack<T, N> out;
#pragma unroll
            for (int i = 0; i < N; ++i) out.set(i, given ? a.scale * in[r][k].get(i) : 0.f);       // no negative zeros
            if (piece < per_row) out.store(to + (int64_t)piece * N);
        }
    }
}

// The same for rows that start anywhere: pieces of 16 bytes where the result's memory has such a boundary, put together from the aligned words around the
// table's entries (of those that hold one of the row), entry by entry at a row's ends.
template <typename T, typename P>
__global__ void __launch_bounds__(256, 4) embed_ragged_kernel(const EmbedArgs a, int per_row, int rows, int lanes_log2) {
    constexpr int kRows = 2, kPieces = 2, N = 16 / sizeof(T), kLoads = (N * (int)sizeof(P) + 15) / 16;
    pdl_wait();
    const int lane = threadIdx.x & 31, l = lane & ((1 << lanes_log2) - 1), sub = lane >> lanes_log2, at_once = 32 >> lanes_log2;
    const int64_t row0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * kRows * at_once + sub;
    const int piece0 = blockIdx.y * (kPieces << lanes_log2) + l;
    uint4 in[kRows][kPieces][kLoads + 1];
    int id[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) id[r] = row0 + r * at_once < rows ? a.tokens[row0 + r * at_once] : -1;
    auto given = [&](int r) { return (uint32_t)id[r] < (uint64_t)a.vocab; };
    auto to = [&](int r) { return static_cast<T *>(a.y.data) + a.y.at(row0 + r * at_once); };
    auto table = [&](int r) { return static_cast<const P *>(a.table) + (a.ldt ? (uint32_t)(row0 + r * at_once) / (uint32_t)a.n * a.ldt : 0) + id[r] * a.cols; };
    auto first = [&](int r, int k) { return (int64_t)(piece0 + (k << lanes_log2)) * N - (int)(reinterpret_cast<uintptr_t>(to(r)) % 16 / sizeof(T)); };      // entry of a piece
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
#pragma unroll
            for (int i = 0; i <= kLoads; ++i) {
                in[r][k][i] = make_uint4(0, 0, 0, 0);
                if (!given(r)) continue;
                const uintptr_t begin = reinterpret_cast<uintptr_t>(table(r)), word = ((begin + first(r, k) * (int)sizeof(P)) & ~(uintptr_t)15) + i * 16;
                if (word + 16 > begin && word < begin + a.cols * sizeof(P)) in[r][k][i] = *reinterpret_cast<const uint4 *>(word);
            }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (row0 + r * at_once >= rows) break;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int64_t c = first(r, k);
            if (c >= a.cols || piece0 + (k << lanes_log2) >= per_row) continue;
            const unsigned off = given(r) ? (unsigned)((reinterpret_cast<uintptr_t>(table(r)) + c * (int)sizeof(P)) & 15) : 0u;
            Pack<P, N> e;
            uint4 w[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) w[i] = shifted<sizeof(P)>(in[r][k][i], in[r][k][i + 1], off);
#pragma unroll
            for (int i = 0; i < Pack<P, N>::kWords; ++i) {
                const uint32_t q[4] = {w[i / 4].x, w[i / 4].y, w[i / 4].z, w[i / 4].w};
                e.w[i] = q[i % 4];
            }
            Pack<T, N> out;
#pragma unroll
            for (int i = 0; i < N; ++i) out.set(i, given(r) ? a.scale * e.get(i) : 0.f);
            T *at = to(r) + c;
            if (c >= 0 && c + N <= a.cols) {
                out.store(at);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (c + i >= 0 && c + i < a.cols) put(at + i, out.get(i));
            }
        }
    }
}

template <typename T, typename P>
cudaError_t embed(const EmbedArgs &a, cudaStream_t s) {
    constexpr int N = sizeof(T) + sizeof(P) == 4 ? 8 : 4;               // 16 bytes of the wider type
    const bool vectors = a.cols % N == 0 && aligned_to(a.y, a.m, a.n, sizeof(T), N * sizeof(T)) && reinterpret_cast<uintptr_t>(a.table) % (N * sizeof(P)) == 0 && a.ldt % N == 0;
    const int64_t rows = a.m * a.n, per_row = vectors ? a.cols / N : a.cols / (16 / (int)sizeof(T)) + 2;
    int lanes_log2 = 0;
    while (lanes_log2 < 5 && (1 << lanes_log2) < per_row) ++lanes_log2;
    const int64_t rows_per_block = 8 * (vectors ? 4 : 2) * (32 >> lanes_log2);
    const dim3 grid((unsigned)((rows + rows_per_block - 1) / rows_per_block), (unsigned)((per_row + (2 << lanes_log2) - 1) / (2 << lanes_log2)));
    auto *kernel = vectors ? embed_kernel<T, P, N> : embed_ragged_kernel<T, P>;
    return launch_chained(kernel, grid, dim3(256), 0, s, true, a, (int)per_row, (int)rows, lanes_log2);
}

// ---- gradient

constexpr int kOrderWarps = 16, kOrderThreads = 32 * kOrderWarps;
constexpr int kClassRows = 1024;                     // rows of a class at most
constexpr int kQueue = 512;                          // tokens of its class that a warp notes on its way: the row, and in 22 bits which of its stretch
constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kZeroSlice = 4096;                     // columns of a warp that writes zeros, and about how many bytes in all: with 16 KB the ticket is what all
constexpr int kZeroBytes = 48 << 10;                 // wait for (8 tables of 32000 x 4096 in bfloat16, 2.1 GB: 460 us, 320 with 32 KB)
constexpr int kRun = 32;                             // sorted positions of a warp
constexpr int kCopied = 8;                           // rows of dy that a warp asks for at a time; it has two such lots in shared memory
constexpr int kSliceBytes = 512, kPitch = kSliceBytes + 16;        // of a row of dy: a warp's, and where it lies in shared memory

// The rows of class c: c, c + count, c + 2 count and so on, so that neighbouring ids (the frequent ones, say) belong to different classes.
struct Classes {
    int log2_count, rows;                            // of the classes; rows of one, at most
    __host__ __device__ int count() const { return 1 << log2_count; }
    __host__ __device__ int64_t starts() const { return rows + 1; }
    __device__ __forceinline__ uint32_t row(uint32_t id) const { return id >> log2_count; }
    __device__ __forceinline__ uint32_t cls(uint32_t id) const { return id & (uint32_t)(count() - 1); }
};

// Every class's block reads all of a worker's tokens: no more classes than there are SMs (of this design, so that the workspace's size needs no device),
// unless a class's counters would not fit in shared memory.
Classes classes_of(int m, int64_t vocab) {
    Classes c = {};
    while ((((vocab - 1) >> c.log2_count) + 1 > kClassRows || ((int64_t)m << c.log2_count) < 128) && ((int64_t)2 << c.log2_count) <= vocab) ++c.log2_count;
    c.rows = (int)(((vocab - 1) >> c.log2_count) + 1);
    return c;
}

struct Token { int position, id; };

// What lies where in the workspace.
struct Plan {
    int64_t start, count, list, parts, bytes;
};
int64_t runs_of(int64_t n) { return (n + kRun - 1) / kRun; }
Plan plan_embed(int m, int64_t n, int64_t vocab, int64_t cols) {
    const Classes c = classes_of(m, vocab);
    auto up = [](int64_t v) { return (v + 255) / 256 * 256; };
    Plan p = {};
    p.count = up((int64_t)m * c.count() * c.starts() * 4);
    p.list = p.count + up((int64_t)m * 8);
    p.parts = p.list + up(m * n * 8);
    p.bytes = p.parts + 2 * m * runs_of(n) * cols * 4;
    return p;
}

// start[worker][class][row]: where the positions of the class's row begin in list[worker]; one more entry ends the last row's.
// count[worker]: all of them, and the next kernel's ticket.
__global__ void __launch_bounds__(kOrderThreads) embed_order_kernel(const int32_t *tokens, int64_t n, int64_t vocab, const Classes c, int *start, int2 *count, Token *list) {
    constexpr int kAtOnce = 16, kTurn = 32 * kAtOnce;
    extern __shared__ int counters[];                // [warp][row]
    __shared__ int lower_of[kOrderWarps], sum_of[kOrderWarps];
    __shared__ uint32_t queue[kOrderWarps][kQueue];
    pdl_wait();
    pdl_launch_dependents();
    const int worker = blockIdx.y, cls = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    tokens += worker * n;
    list += worker * n;
    start += ((int64_t)worker * c.count() + cls) * c.starts();
    for (int i = threadIdx.x; i < kOrderWarps * c.rows; i += kOrderThreads) counters[i] = 0;
    __syncthreads();
    const uint32_t stretch = (uint32_t)((n + kOrderWarps * 32 - 1) / (kOrderWarps * 32)) * 32;
    const uint32_t from = (uint32_t)min(n, (int64_t)warp * stretch), to = (uint32_t)min(n, (int64_t)from + stretch);
    int *mine = counters + warp * c.rows;
    auto load = [&](uint32_t t0, uint32_t (&id)[kAtOnce]) {
        const int32_t *at = tokens + t0 + lane;
        if (to - t0 >= kTurn) {
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) id[k] = (uint32_t)at[k * 32];
        } else {
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) id[k] = k * 32 + lane < to - t0 ? (uint32_t)at[k * 32] : 0xffffffffu;
        }
    };
    const uint32_t words = (uint32_t)vocab;
    int lower = 0, queued = 0;
    for (uint32_t t0 = from; t0 < to; t0 += kTurn) {
        uint32_t id[kAtOnce];
        load(t0, id);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const bool own = id[k] < words && c.cls(id[k]) == (uint32_t)cls;
            lower += id[k] < words && c.cls(id[k]) < (uint32_t)cls;
            const unsigned owners = __ballot_sync(0xffffffffu, own);
            if (owners) {
                const int at = queued + __popc(owners & ((1u << lane) - 1));
                if (own) atomicAdd(mine + c.row(id[k]), 1);
                if (own && at < kQueue) queue[warp][at] = c.row(id[k]) << 22 | (t0 - from + k * 32 + lane);
                queued += __popc(owners);
            }
        }
    }
    lower = __reduce_add_sync(0xffffffffu, lower);
    if (lane == 0) lower_of[warp] = lower;
    __syncthreads();
    // Where each row begins, and each warp's part of it: two rows a thread.
    static_assert(kClassRows <= 2 * kOrderThreads, "rows of a thread");
    int before = 0, all[2] = {};
#pragma unroll
    for (int w = 0; w < kOrderWarps; ++w) before += lower_of[w];
    const int row0 = threadIdx.x * 2;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (row0 + k < c.rows)
#pragma unroll
            for (int w = 0; w < kOrderWarps; ++w) all[k] += counters[w * c.rows + row0 + k];
    int scan = all[0] + all[1];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, scan, d);
        if (lane >= d) scan += v;
    }
    if (lane == 31) sum_of[warp] = scan;
    __syncthreads();
    for (int w = 0; w < warp; ++w) before += sum_of[w];
    before += scan - all[0] - all[1];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (row0 + k < c.rows) {
            start[row0 + k] = before;
#pragma unroll
            for (int w = 0; w < kOrderWarps; ++w) {
                const int v = counters[w * c.rows + row0 + k];
                counters[w * c.rows + row0 + k] = before;
                before += v;
            }
            if (row0 + k + 1 == c.rows) {
                start[c.rows] = before;
                if (cls + 1 == c.count()) count[worker] = make_int2(before, 0);
            }
        }
    __syncthreads();
    auto place = [&](bool own, Token t) {                 // a warp's next tokens, in their order
        if (!__any_sync(0xffffffffu, own)) return;
        const int row = own ? (int)c.row(t.id) : -1;
        const unsigned same = __match_any_sync(0xffffffffu, row), below = same & ((1u << lane) - 1);
        const int at = own ? mine[row] + __popc(below) : 0;
        __syncwarp();
        if (own) {
            list[at] = t;
            if (below == 0) mine[row] = at + __popc(same);
        }
        __syncwarp();
    };
    static_assert(kClassRows <= 1 << 10, "bits of a row");
    if (queued <= kQueue && stretch <= 1u << 22) {
        for (int k = 0; k < queued; k += 32) {
            const uint32_t q = k + lane < queued ? queue[warp][k + lane] : 0;
            place(k + lane < queued, Token{(int)(from + (q & 0x3fffffu)), (int)(q >> 22 << c.log2_count | cls)});
        }
        return;
    }
    for (uint32_t t0 = from; t0 < to; t0 += kTurn) {      // a frequent id
        uint32_t id[kAtOnce];
        load(t0, id);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) place(id[k] < words && c.cls(id[k]) == (uint32_t)cls, Token{(int)(t0 + k * 32 + lane), (int)id[k]});
    }
}

// A lane's N of a warp's columns: neighbours where all rows are aligned (VECTORS), else every 32nd.
template <int N, bool VECTORS>
__device__ __forceinline__ int column(int lane, int k) { return VECTORS ? lane * N + k : lane + 32 * k; }

template <int N, bool VECTORS, typename P>
__device__ __forceinline__ void store_columns(const float (&sum)[N], P *row, int lane, int cols, float scale, bool add) {
    if constexpr (VECTORS) {
        if (lane * N >= cols) return;
        Pack<P, N> e;
        if (add) e.load(row + lane * N);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if constexpr (sizeof(P) == 2) {                          // both halves of a word are read before one is set
                if (k & 1) continue;
                const float lo = add ? fmaf(scale, sum[k], e.get(k)) : scale * sum[k], hi = add ? fmaf(scale, sum[k + 1], e.get(k + 1)) : scale * sum[k + 1];
                e.set(k, lo);
                e.set(k + 1, hi);
            } else {
                e.set(k, add ? fmaf(scale, sum[k], e.get(k)) : scale * sum[k]);
            }
        }
        e.store(row + lane * N);
    } else {
        float old[N] = {};
        if (add)
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (lane + 32 * k < cols) old[k] = value_of(row + lane + 32 * k);
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (lane + 32 * k < cols) put(row + lane + 32 * k, add ? fmaf(scale, sum[k], old[k]) : scale * sum[k]);
    }
}

// Zeros to n entries, by a warp: 16 bytes a store, of rows that start anywhere where they fit.
template <bool VECTORS, typename P>
__device__ __forceinline__ void zero_entries(P *a, int n, int lane) {
    constexpr int kPer = 16 / sizeof(P);
    if (!VECTORS) {
        const int head = min(n, (int)((16 - reinterpret_cast<uintptr_t>(a) % 16) % 16 / sizeof(P)));
        if (lane < head) a[lane] = P(0.f);
        a += head;
        n -= head;
    }
    const int whole = n / kPer;
#pragma unroll 4
    for (int i = lane; i < whole; i += 32) reinterpret_cast<uint4 *>(a)[i] = make_uint4(0, 0, 0, 0);
    if (!VECTORS && lane < n - whole * kPer) a[whole * kPer + lane] = P(0.f);
}

__device__ __forceinline__ uint32_t smem_address(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

struct RowsArgs {
    EmbedGradArgs a;
    Classes c;
    const int *start;
    int2 *count;
    const Token *list;
    float *parts;                                    // [worker][run][2][cols]: what the run has of the row it begins in the middle of, and of the one it ends in
    int64_t runs;                                    // of a worker, at most
    int followed;                                    // the third kernel comes after the second
    int slices, zero_rows, zero_chunks, zero_slices; // of a worker: slices of columns; groups of zero_rows rows, and their slices
};

// blockIdx.y: the worker.  Its warps take runs of sorted positions in turn, then, whoever is free, groups of rows to write zeros to.  The rows of dy are copied
// to shared memory (from 16-byte boundaries; what a lane did not copy itself it reads only where rows are not aligned), one lot ahead of the sums.
template <typename T, typename P, bool VECTORS>
__global__ void __launch_bounds__(kThreads, 3) embed_rows_kernel(const RowsArgs r) {
    constexpr int N = 16 / sizeof(T), kSlice = 32 * N;
    extern __shared__ __align__(16) uint8_t copied[];
    pdl_wait();
    if (r.followed) pdl_launch_dependents();              // never the next call's: a call's last kernel lets nothing start before its end
    const EmbedGradArgs &a = r.a;
    const Classes c = r.c;
    const int lane = threadIdx.x & 31, worker = blockIdx.y;
    const uint32_t warp = blockIdx.x * kWarps + (threadIdx.x >> 5), warps = gridDim.x * kWarps;
    P *table = static_cast<P *>(a.dtable) + worker * a.ldt;
    const Token *list = r.list + worker * a.n;
    const int count = __ldcg(&r.count[worker].x);
    uint8_t *rows = copied + (threadIdx.x >> 5) * 2 * kCopied * kPitch;
    const uint32_t tasks = (uint32_t)((count + kRun - 1) / kRun) * r.slices;
    // the run's positions, as many before and as many behind them
    Token ahead[3];
    auto ask = [&](uint32_t task) {
        const int p0 = (int)(task / (uint32_t)r.slices) * kRun;
#pragma unroll
        for (int h = 0; h < 3; ++h) {
            const int p = p0 + (h - 1) * kRun + lane;
            ahead[h] = task < tasks && p >= 0 && p < count ? list[p] : Token{0, -1};
        }
    };
    ask(warp);
    for (uint32_t task = warp; task < tasks; task += warps) {
        const uint32_t run = task / (uint32_t)r.slices, slice = task - run * r.slices;
        const int64_t col0 = (int64_t)slice * kSlice;
        const int p0 = run * kRun, cols = (int)min((int64_t)kSlice, a.cols - col0);
        const T *dy = static_cast<const T *>(a.dy.data) + worker * a.dy.group + col0;
        const Token mine[2] = {ahead[1], ahead[2]};
        const int earlier = ahead[0].id;
        ask(task + warps);
        const int head = __shfl_sync(0xffffffffu, mine[0].id, 0), tail = __shfl_sync(0xffffffffu, mine[0].id, 31);
        const unsigned heads = __ballot_sync(0xffffffffu, mine[0].id == head), tails = __ballot_sync(0xffffffffu, mine[0].id == tail);
        const unsigned behind = __ballot_sync(0xffffffffu, tail >= 0 && mine[1].id == tail), before = __ballot_sync(0xffffffffu, earlier == head);
        int k = 0, end = min(kRun, count - p0);                    // positions that this warp sums
        // The row that the run begins in began before.  It is a long one if the position kRun before its last one here is its own, too, or it goes on.
        const bool continued = before >> 31, parted = continued && (heads == 0xffffffffu || (before >> (__popc(heads) - 1) & 1));
        if (continued && !parted) k = __popc(heads);
        // The row that the run ends in goes on, and is a long one.
        const bool goes_on = behind & 1, long_tail = goes_on && ((continued && tail == head) || __popc(tails) + __popc(behind) > kRun);
        if (goes_on && !long_tail) end += __popc(behind);
        const int next0 = __shfl_down_sync(0xffffffffu, mine[0].id, 1), next1 = __shfl_down_sync(0xffffffffu, mine[1].id, 1), middle = __shfl_sync(0xffffffffu, mine[1].id, 0);
        const unsigned ends0 = __ballot_sync(0xffffffffu, (lane == 31 ? middle : next0) != mine[0].id), ends1 = __ballot_sync(0xffffffffu, lane == 31 || next1 != mine[1].id);
        const uint64_t ends = ((uint64_t)ends1 << 32 | ends0) | (uint64_t)1 << (end - 1);              // last positions of a row, or of this warp
        float *parts = r.parts + ((int64_t)worker * r.runs + run) * 2 * a.cols + col0;
        auto position = [&](int at) {
            const int low = __shfl_sync(0xffffffffu, mine[0].position, at & 31), high = __shfl_sync(0xffffffffu, mine[1].position, at & 31);
            return at < kRun ? low : high;
        };
        auto copy = [&](int from, int lot) {                       // the next kCopied rows
            if (!VECTORS) __syncwarp();                            // what lay there has been read
#pragma unroll
            for (int q = 0; q < kCopied; ++q) {
                const uintptr_t row = reinterpret_cast<uintptr_t>(dy + position(from + q) * a.dy.row);
                const int off = VECTORS ? 0 : (int)(row & 15), bytes = off + cols * (int)sizeof(T);
                const uint32_t to = smem_address(rows + (lot * kCopied + q) * kPitch);
                if (from + q >= end) break;
                if (lane * 16 < bytes) cp_async<16>(to + lane * 16, reinterpret_cast<const void *>(row - off + lane * 16));
                if (!VECTORS && lane == 0 && bytes > kSliceBytes) cp_async<16>(to + kSliceBytes, reinterpret_cast<const void *>(row - off + kSliceBytes));
            }
            cp_async_commit();
        };
        float sum[N] = {};
        int lot = 0;
        if (k < end) copy(k, 0);
        for (; k < end; lot ^= 1) {
            copy(k + kCopied, lot ^ 1);                            // nothing, at the end
            cp_async_wait<1>();
            if (!VECTORS) __syncwarp();
            const int here = min(kCopied, end - k);
#pragma unroll 2
            for (int q = 0; q < here; ++q, ++k) {
                const uint8_t *from = rows + (lot * kCopied + q) * kPitch;
                if constexpr (VECTORS) {
                    Pack<T, N> e;
                    e.load(reinterpret_cast<const T *>(from) + lane * N);
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[i] += e.get(i);
                } else {
                    const T *entries = reinterpret_cast<const T *>(from + (reinterpret_cast<uintptr_t>(dy + position(k) * a.dy.row) & 15)) + lane;
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[i] += value_of(entries + 32 * i);
                }
                if (!(ends >> k & 1)) continue;
                const int id = __shfl_sync(0xffffffffu, mine[0].id, min(k, 31));            // of a row that begins in the run
                const bool first = parted && id == head, last = long_tail && id == tail;
                if (first || last) {                               // of a run that lies within a row there is one part, the first
                    float *to = parts + (first ? 0 : a.cols);
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (column<N, VECTORS>(lane, i) < cols) to[column<N, VECTORS>(lane, i)] = sum[i];
                } else {
                    store_columns<N, VECTORS>(sum, table + id * a.cols + col0, lane, cols, a.scale, a.add);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = 0.f;
            }
        }
        cp_async_wait<0>();
        __syncwarp();
    }
    if (a.add) return;
    const uint32_t zeros = (uint32_t)r.zero_chunks * r.zero_slices;
    const int *start = r.start + (int64_t)worker * c.count() * c.starts();
    for (;;) {
        uint32_t task = 0;
        if (lane == 0) task = atomicAdd(reinterpret_cast<unsigned *>(&r.count[worker].y), 1u);
        task = __shfl_sync(0xffffffffu, task, 0);
        if (task >= zeros) break;
        const uint32_t chunk = task / (uint32_t)r.zero_slices, slice = task - chunk * r.zero_slices, id = chunk * r.zero_rows + lane;
        const int64_t col0 = (int64_t)slice * kZeroSlice;
        const int cols = (int)min((int64_t)kZeroSlice, a.cols - col0);
        const int *s = start + c.cls(id) * c.starts() + c.row(id);
        unsigned none = __ballot_sync(0xffffffffu, lane < r.zero_rows && id < (uint32_t)a.vocab && __ldcg(s) == __ldcg(s + 1));
        P *first = table + (int64_t)chunk * r.zero_rows * a.cols + col0;
        while (none) {
            const int at = __ffs(none) - 1;
            const unsigned others = ~(none >> at);
            // whole rows that follow one another are one stretch
            const int together = r.zero_slices > 1 ? 1 : others ? __ffs(others) - 1 : 32;
            zero_entries<VECTORS>(first + at * a.cols, together * cols, lane);
            none &= together + at >= 32 ? 0u : ~0u << (at + together);
        }
    }
}

// Rows of more than kRun positions: a block looks for those that begin in kChecked runs and adds their parts, 64 columns of them.  A warp takes a row, or, of more
// than kOwnParts parts, all warps an equal share of it, joined in their order (65536 tokens, 131072 words by 2048 columns, a sixteenth of the tokens one word: 255 us
// in all, by a warp for every row 272).
constexpr int kChecked = 32, kOwnParts = 32;
template <typename P>
__global__ void __launch_bounds__(kThreads) embed_parts_kernel(const RowsArgs r, int slices) {
    constexpr int N = 2, kSlice = 32 * N, kAtOnce = 16;
    __shared__ LongSum shares[kWarps][kSlice];
    pdl_wait();
    const EmbedGradArgs &a = r.a;
    const Classes c = r.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, worker = blockIdx.y;
    const Token *list = r.list + worker * a.n;
    const int *start = r.start + (int64_t)worker * c.count() * c.starts();
    const int count = r.count[worker].x;
    const uint32_t runs = (count + kRun - 1) / kRun, tasks = (runs + kChecked - 1) / kChecked * slices;
    for (uint32_t task = blockIdx.x; task < tasks; task += gridDim.x) {
        const uint32_t group = task / (uint32_t)slices, slice = task - group * slices, mine = group * kChecked + lane;
        int id = -1, from = 0, of_row = 0;
        if (mine < runs) {
            id = list[min(count, (int)(mine + 1) * kRun) - 1].id;
            const int *s = start + c.cls(id) * c.starts() + c.row(id);
            from = s[0], of_row = s[1] - s[0];
        }
        const int64_t col0 = (int64_t)slice * kSlice;
        const int cols = (int)min((int64_t)kSlice, a.cols - col0);
        const float *parts = r.parts + (int64_t)worker * r.runs * 2 * a.cols + col0;
        // the row's parts in runs k0 to last
        auto add = [&](LongSum (&total)[N], uint32_t k0, uint32_t last) {
            for (; k0 <= last; k0 += kAtOnce) {
                float v[kAtOnce][N];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i) v[k][i] = k0 + k <= last && lane + 32 * i < cols ? parts[(int64_t)(k0 + k) * 2 * a.cols + lane + 32 * i] : 0.f;
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
                    for (int i = 0; i < N; ++i) total[i].add(v[k][i]);
            }
        };
        auto store = [&](const LongSum (&total)[N], int row) {
            float sum[N];
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = total[i].sum;
            store_columns<N, false>(sum, static_cast<P *>(a.dtable) + worker * a.ldt + row * a.cols + col0, lane, cols, a.scale, a.add);
        };
        int turn = 0;
        for (unsigned found = __ballot_sync(0xffffffffu, of_row > kRun && from / kRun == (int)mine); found; found &= found - 1, ++turn) {
            const int at = __ffs(found) - 1, row = __shfl_sync(0xffffffffu, id, at);
            const uint32_t run = group * kChecked + at, last = (__shfl_sync(0xffffffffu, from + of_row, at) - 1) / kRun, more = last - run;
            const bool shared = more > kOwnParts, own = turn % kWarps == warp;
            if (!shared && !own) continue;
            LongSum total[N];
            if (own)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (lane + 32 * i < cols) total[i].sum = parts[((int64_t)run * 2 + 1) * a.cols + lane + 32 * i];
            if (!shared) {
                add(total, run + 1, last);
                store(total, row);
                continue;
            }
            LongSum share[N];
            add(share, run + 1 + (uint32_t)((uint64_t)more * warp / kWarps), run + (uint32_t)((uint64_t)more * (warp + 1) / kWarps));
#pragma unroll
            for (int i = 0; i < N; ++i) shares[warp][lane + 32 * i] = share[i];
            __syncthreads();
            if (own) {
                for (int w = 0; w < kWarps; ++w)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const LongSum of_warp = shares[w][lane + 32 * i];
                        total[i].add(of_warp.sum);
                        total[i].add(-of_warp.lost);
                    }
                store(total, row);
            }
            __syncthreads();
        }
    }
}

template <typename T, typename P, bool VECTORS>
cudaError_t sum_rows(RowsArgs r, cudaStream_t s) {
    constexpr int kSmem = kWarps * 2 * kCopied * kPitch;
    constexpr int kSlice = kSliceBytes / (int)sizeof(T);
    static PerDeviceOnce once;
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (once.need(device)) {
        e = cudaFuncSetAttribute(embed_rows_kernel<T, P, VECTORS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return e;
        once.mark(device);
    }
    r.slices = (int)((r.a.cols + kSlice - 1) / kSlice);
    const int64_t runs = runs_of(r.a.n) * r.slices, zeros = (int64_t)r.zero_chunks * r.zero_slices;
    auto blocks_for = [&](int64_t warps, int per_sm) {                 // of one worker: so many blocks an SM for all of them
        const int64_t all = (warps + kWarps - 1) / kWarps, most = (148 * per_sm + r.a.m - 1) / r.a.m;
        return (unsigned)(all < most ? (all > 0 ? all : 1) : most);
    };
    e = launch_chained(embed_rows_kernel<T, P, VECTORS>, dim3(blocks_for(zeros > runs ? zeros : runs, 3), r.a.m), dim3(kThreads), kSmem, s, true, r);
    if (e != cudaSuccess) return e;
    if (!r.followed) return cudaSuccess;                               // no row of more than a run
    const int slices = (int)((r.a.cols + 63) / 64);
    return launch_chained(embed_parts_kernel<P>, dim3(blocks_for((runs_of(r.a.n) + kChecked - 1) / kChecked * slices * kWarps, 6), r.a.m), dim3(kThreads), 0, s, true, r, slices);
}

template <typename T, typename P>
cudaError_t embed_gradient(const EmbedGradArgs &a, cudaStream_t s) {
    const Plan p = plan_embed(a.m, a.n, a.vocab, a.cols);
    const Classes c = classes_of(a.m, a.vocab);
    uint8_t *ws = static_cast<uint8_t *>(a.workspace);
    int *start = reinterpret_cast<int *>(ws + p.start);
    int2 *count = reinterpret_cast<int2 *>(ws + p.count);
    Token *list = reinterpret_cast<Token *>(ws + p.list);
    static PerDeviceOnce once;
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (once.need(device)) {
        e = cudaFuncSetAttribute(embed_order_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kOrderWarps * kClassRows * 4);
        if (e != cudaSuccess) return e;
        once.mark(device);
    }
    e = launch_chained(embed_order_kernel, dim3(c.count(), a.m), dim3(kOrderThreads), (size_t)kOrderWarps * c.rows * 4, s, true, a.tokens, a.n, a.vocab, c, start, count, list);
    if (e != cudaSuccess) return e;
    RowsArgs r = {a, c, start, count, list, reinterpret_cast<float *>(ws + p.parts), runs_of(a.n), a.n > kRun, 0, 0, 0, 0};
    r.zero_slices = (int)((a.cols + kZeroSlice - 1) / kZeroSlice);
    const int64_t rows = kZeroBytes / ((a.cols < kZeroSlice ? a.cols : kZeroSlice) * (int)sizeof(P));
    const int64_t shares = (int64_t)a.m * a.vocab * r.zero_slices / (148 * 3 * kWarps) + 1;           // so that every warp has some
    r.zero_rows = (int)(rows < 1 ? 1 : rows < 32 ? rows : 32);
    if (shares < r.zero_rows) r.zero_rows = (int)shares;
    r.zero_chunks = a.add ? 0 : (int)((a.vocab + r.zero_rows - 1) / r.zero_rows);
    const bool vectors = a.cols % 8 == 0 && aligned_to(a.dy, a.m, a.n, sizeof(T), 16) && reinterpret_cast<uintptr_t>(a.dtable) % 16 == 0 && (a.m <= 1 || a.ldt * sizeof(P) % 16 == 0);
    return vectors ? sum_rows<T, P, true>(r, s) : sum_rows<T, P, false>(r, s);
}

}  // namespace

cudaError_t launch_embed(int type, int param_type, const EmbedArgs &a, cudaStream_t s) {
    if (type == ZENO_F32) return param_type == ZENO_F32 ? embed<float, float>(a, s) : embed<float, __nv_bfloat16>(a, s);
    return param_type == ZENO_F32 ? embed<__nv_bfloat16, float>(a, s) : embed<__nv_bfloat16, __nv_bfloat16>(a, s);
}

int64_t embed_gradient_workspace(int m, int64_t n, int64_t vocab, int64_t cols) { return plan_embed(m, n, vocab, cols).bytes; }

// A warp's tasks are counted in 32 bits.
bool embed_gradient_fits(int64_t n, int64_t vocab, int64_t cols) {
    const int64_t limit = (int64_t)1 << 31;
    return runs_of(n) * ((cols + 63) / 64) < limit && (vocab + 1) * ((cols + kZeroSlice - 1) / kZeroSlice) < limit;
}

cudaError_t launch_embed_gradient(int type, int param_type, const EmbedGradArgs &a, cudaStream_t s) {
    if (type == ZENO_F32) return param_type == ZENO_F32 ? embed_gradient<float, float>(a, s) : embed_gradient<float, __nv_bfloat16>(a, s);
    return param_type == ZENO_F32 ? embed_gradient<__nv_bfloat16, float>(a, s) : embed_gradient<__nv_bfloat16, __nv_bfloat16>(a, s);
}

}  // namespace zeno

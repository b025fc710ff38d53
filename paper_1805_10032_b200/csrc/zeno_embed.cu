// A language model's embedding, y_t = scale E[id_t], and its gradient for every worker, dE[v] = scale sum over the tokens with id v of dy_t.
//
// Forward: a thread gathers 8 neighbouring entries (or one, of rows that start anywhere); bound by memory.
// Backward: every row of the table is written once, mostly zeros, and no row is summed by atomics.  A first kernel sorts each worker's token positions by
// id: a block per class of ids (id mod classes) counts what each of its warps finds in a stretch of the tokens, and places the positions, rows in order, positions
// in order within a row.  A second one walks over the rows, a warp to 512 columns of a row; rows with many tokens are shared by a block's warps.
#include "zeno_operators.h"

namespace zeno {

namespace {

template <typename T, int N>
struct alignas(sizeof(T) * N <= 16 ? sizeof(T) * N : 16) Pack {
    T v[N];
};

template <typename T, typename P, int N>
__global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a, int per_row, int64_t rows, int rows_per_block) {
    constexpr int kAtOnce = 4;
    pdl_wait();
    const int64_t row0 = (int64_t)blockIdx.x * rows_per_block;
    const int here = (int)min((int64_t)rows_per_block, rows - row0), pieces = here * per_row;
    for (int q0 = threadIdx.x; q0 < pieces; q0 += 256 * kAtOnce) {
        Pack<P, N> in[kAtOnce];
        T *to[kAtOnce];
        bool given[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int q = q0 + k * 256;
            if (q >= pieces) break;
            const int r = q / per_row;
            const int64_t row = row0 + r, c = (int64_t)(q - r * per_row) * N;
            const int id = a.tokens[row];
            to[k] = static_cast<T *>(a.y.data) + a.y.at(row) + c;
            given[k] = (uint32_t)id < (uint64_t)a.vocab;
            if (given[k]) in[k] = *reinterpret_cast<const Pack<P, N> *>(static_cast<const P *>(a.table) + (a.ldt ? row / a.n * a.ldt : 0) + id * a.cols + c);
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            if (q0 + k * 256 >= pieces) break;
            Pack<T, N> out;
#pragma unroll
            for (int i = 0; i < N; ++i) put(out.v + i, given[k] ? a.scale * value_of(in[k].v + i) : 0.f);
            *reinterpret_cast<Pack<T, N> *>(to[k]) = out;
        }
    }
}

template <typename T, typename P>
cudaError_t embed(const EmbedArgs &a, cudaStream_t s) {
    const int64_t rows = a.m * a.n;
    const bool vectors = a.cols % 8 == 0 && aligned_to(a.y, a.m, a.n, sizeof(T), 16) && reinterpret_cast<uintptr_t>(a.table) % 16 == 0 && a.ldt % 8 == 0;
    const int64_t per_row = vectors ? a.cols / 8 : a.cols;
    int64_t rows_per_block = 1024 / per_row;
    if (rows_per_block < 1) rows_per_block = 1;
    const int64_t blocks = (rows + rows_per_block - 1) / rows_per_block;
    auto *kernel = vectors ? embed_kernel<T, P, 8> : embed_kernel<T, P, 1>;
    return launch_chained(kernel, dim3((unsigned)blocks), dim3(256), 0, s, true, a, (int)per_row, rows, (int)rows_per_block);
}

// ---- gradient

constexpr int kWarps = 16, kThreads = 32 * kWarps;
constexpr int kClassRows = 1024;                     // rows of a class at most
constexpr int kSlice = 512;                          // columns of a warp
constexpr int kChain = 64;                           // tokens summed by one chain of additions, and by one warp

struct Classes {
    int count, rows, slices;                         // classes; rows of one, at most
    __host__ __device__ int64_t starts() const { return rows + 1; }
};

// Classes: as many as make four blocks an SM, and a class's counters fit in shared memory.  The count of SMs is this design's.
Classes classes_of(int m, int64_t vocab, int64_t cols) {
    Classes c;
    c.slices = (int)((cols + kSlice - 1) / kSlice);
    int64_t count = 592 / ((int64_t)m * c.slices);
    if (count < (vocab + kClassRows - 1) / kClassRows) count = (vocab + kClassRows - 1) / kClassRows;
    if (count > vocab) count = vocab;
    c.count = (int)count;
    c.rows = (int)((vocab + count - 1) / count);
    return c;
}

// start[worker][class][row]: where the positions of the class's row begin in list[worker]; one more entry ends the last row's.
__global__ void __launch_bounds__(kThreads) embed_order_kernel(const int32_t *tokens, int64_t n, int64_t vocab, Classes c, int *start, int *list) {
    extern __shared__ int counters[];                // [warp][row]
    __shared__ int lower_of[kWarps], sum_of[kWarps];
    pdl_wait();
    pdl_launch_dependents();
    const int worker = blockIdx.y, cls = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    tokens += worker * n;
    list += worker * n;
    start += ((int64_t)worker * c.count + cls) * c.starts();
    for (int i = threadIdx.x; i < kWarps * c.rows; i += kThreads) counters[i] = 0;
    __syncthreads();
    const int64_t stretch = (n + kWarps * 128 - 1) / (kWarps * 128) * 128, from = warp * stretch, to = min(n, from + stretch);
    int *mine = counters + warp * c.rows;
    const uint32_t classes = c.count;
    int lower = 0;
    for (int64_t t0 = from; t0 < to; t0 += 128) {
        int id[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) id[k] = t0 + k * 32 + lane < to ? tokens[t0 + k * 32 + lane] : -1;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool given = (uint32_t)id[k] < (uint64_t)vocab;
            const uint32_t row = (uint32_t)id[k] / classes, in = (uint32_t)id[k] - row * classes;
            lower += __popc(__ballot_sync(0xffffffffu, given && in < (uint32_t)cls));
            if (given && in == (uint32_t)cls) atomicAdd(mine + row, 1);
        }
    }
    if (lane == 0) lower_of[warp] = lower;
    __syncthreads();
    // Where each row begins, and each warp's part of it: two rows a thread.
    static_assert(kClassRows <= 2 * kThreads, "rows of a thread");
    int before = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) before += lower_of[w];
    int all[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int row = threadIdx.x * 2 + k;
        if (row < c.rows)
            for (int w = 0; w < kWarps; ++w) {
                const int v = counters[w * c.rows + row];
                counters[w * c.rows + row] = all[k];
                all[k] += v;
            }
    }
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
    for (int k = 0; k < 2; ++k) {
        const int row = threadIdx.x * 2 + k;
        if (row < c.rows) {
            start[row] = before;
            for (int w = 0; w < kWarps; ++w) counters[w * c.rows + row] += before;
            before += all[k];
            if (row + 1 == c.rows) start[row + 1] = before;
        }
    }
    __syncthreads();
    for (int64_t t0 = from; t0 < to; t0 += 128) {
        int id[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) id[k] = t0 + k * 32 + lane < to ? tokens[t0 + k * 32 + lane] : -1;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t row = (uint32_t)id[k] / classes, in = (uint32_t)id[k] - row * classes;
            const bool own = (uint32_t)id[k] < (uint64_t)vocab && in == (uint32_t)cls;
            if (__any_sync(0xffffffffu, own)) {
                const unsigned same = __match_any_sync(0xffffffffu, own ? (int)row : -1), below = same & ((1u << lane) - 1);
                int at = 0;
                if (own) at = mine[row] + __popc(below);
                __syncwarp();
                if (own) {
                    list[at] = (int)(t0 + k * 32 + lane);
                    if (below == 0) mine[row] = at + __popc(same);
                }
                __syncwarp();
            }
        }
    }
}

// 16 columns of a lane: two runs of eight, 256 apart
template <typename T>
__device__ __forceinline__ void add_columns(float (&sum)[16], const T *row, int lane, int cols, bool vectors) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c = h * 256 + lane * 8;
        if (vectors) {
            if (c < cols) {
                Pack<T, 8> e = *reinterpret_cast<const Pack<T, 8> *>(row + c);
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[h * 8 + k] += value_of(e.v + k);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < cols) sum[h * 8 + k] += value_of(row + c + k);
        }
    }
}

// Zeros from a to b, by a warp: 16 bytes a store where they fit.
template <typename P>
__device__ __forceinline__ void zero_entries(P *a, P *b, int lane) {
    constexpr int kPer = 16 / sizeof(P);
    const int head = min((int)(b - a), (int)((16 - reinterpret_cast<uintptr_t>(a) % 16) % 16 / sizeof(P)));
    if (lane < head) a[lane] = P(0.f);
    a += head;
    const int whole = (int)(b - a) / kPer;
    for (int i = lane; i < whole; i += 32) reinterpret_cast<uint4 *>(a)[i] = make_uint4(0, 0, 0, 0);
    a += whole * kPer;
    if (lane < (int)(b - a)) a[lane] = P(0.f);
}

template <typename P>
__device__ __forceinline__ void store_columns(const float (&sum)[16], P *row, int lane, int cols, float scale, bool add, bool vectors) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c = h * 256 + lane * 8;
        if (vectors) {
            if (c >= cols) continue;
            Pack<P, 8> e;
            if (add) e = *reinterpret_cast<const Pack<P, 8> *>(row + c);
#pragma unroll
            for (int k = 0; k < 8; ++k) put(e.v + k, add ? fmaf(scale, sum[h * 8 + k], value_of(e.v + k)) : scale * sum[h * 8 + k]);
            *reinterpret_cast<Pack<P, 8> *>(row + c) = e;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < cols) put(row + c + k, add ? fmaf(scale, sum[h * 8 + k], value_of(row + c + k)) : scale * sum[h * 8 + k]);
        }
    }
}

template <typename T, typename P>
__global__ void __launch_bounds__(kThreads) embed_rows_kernel(const EmbedGradArgs a, const Classes c, const int *start, const int *list, int in_vectors, int out_vectors) {
    __shared__ int starts[kClassRows + 1];
    __shared__ float partial[kWarps][kSlice];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t item = blockIdx.x;
    const int slice = (int)(item % c.slices), cls = (int)(item / c.slices % c.count), worker = (int)(item / c.slices / c.count);
    start += ((int64_t)worker * c.count + cls) * c.starts();
    list += worker * a.n;
    for (int i = threadIdx.x; i <= c.rows; i += kThreads) starts[i] = start[i];
    __syncthreads();
    const int64_t col0 = (int64_t)slice * kSlice;
    const int cols = (int)min((int64_t)kSlice, a.cols - col0), rows = (int)((a.vocab - cls + c.count - 1) / c.count);
    const T *dy = static_cast<const T *>(a.dy.data) + worker * a.dy.group + col0;
    P *out = static_cast<P *>(a.dtable) + worker * a.ldt + cls * a.cols + col0;
    const int64_t pitch = c.count * a.cols;
    for (int row = warp; row < rows; row += kWarps) {
        const int from = starts[row], count = starts[row + 1] - from;
        if (count > kChain) continue;
        P *to = out + row * pitch;
        if (count == 0) {
            if (!a.add) zero_entries(to, to + cols, lane);
            continue;
        }
        float sum[16] = {};
        for (int k0 = 0; k0 < count; k0 += 32) {
            const int position = k0 + lane < count ? list[from + k0 + lane] : 0, here = min(32, count - k0);
#pragma unroll 4
            for (int k = 0; k < here; ++k) add_columns(sum, dy + __shfl_sync(0xffffffffu, position, k) * a.dy.row, lane, cols, in_vectors);
        }
        store_columns(sum, to, lane, cols, a.scale, a.add, out_vectors);
    }
    // Rows of many tokens: every warp sums some, kChain at a time, and their sums are added.
    for (int row = 0; row < rows; ++row) {
        const int from = starts[row], count = starts[row + 1] - from;
        if (count <= kChain) continue;
        LongSum total[16];
        for (int k0 = warp * 8; k0 < count;) {
            float sum[16] = {};
            for (int turns = 0; turns < kChain / 8 && k0 < count; ++turns, k0 += kWarps * 8) {
                const int position = list[from + min(k0 + (lane & 7), count - 1)], here = min(8, count - k0);
#pragma unroll 4
                for (int k = 0; k < here; ++k) add_columns(sum, dy + __shfl_sync(0xffffffffu, position, k) * a.dy.row, lane, cols, in_vectors);
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) total[k].add(sum[k]);
        }
        __syncthreads();                                     // the row before has been read
#pragma unroll
        for (int k = 0; k < 16; ++k) partial[warp][k / 8 * 256 + lane * 8 + k % 8] = total[k].sum;
        __syncthreads();
        if (threadIdx.x < cols) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) s += partial[w][threadIdx.x];
            P *to = out + row * pitch + threadIdx.x;
            put(to, a.add ? fmaf(a.scale, s, value_of(to)) : a.scale * s);
        }
    }
}

template <typename T, typename P>
cudaError_t embed_gradient(const EmbedGradArgs &a, cudaStream_t s) {
    const Classes c = classes_of(a.m, a.vocab, a.cols);
    int *start = static_cast<int *>(a.workspace);
    int *list = start + (int64_t)a.m * c.count * c.starts();
    static PerDeviceOnce once;
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    const size_t smem = (size_t)kWarps * c.rows * 4;
    if (once.need(device)) {
        e = cudaFuncSetAttribute(embed_order_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kWarps * kClassRows * 4);
        if (e != cudaSuccess) return e;
        once.mark(device);
    }
    e = launch_chained(embed_order_kernel, dim3(c.count, a.m), dim3(kThreads), smem, s, true, a.tokens, a.n, a.vocab, c, start, list);
    if (e != cudaSuccess) return e;
    const bool in_vectors = a.cols % 8 == 0 && aligned_to(a.dy, a.m, a.n, sizeof(T), 16);
    const bool out_vectors = a.cols % 8 == 0 && reinterpret_cast<uintptr_t>(a.dtable) % 16 == 0 && (a.m <= 1 || a.ldt * sizeof(P) % 16 == 0);
    return launch_chained(embed_rows_kernel<T, P>, dim3((unsigned)((int64_t)a.m * c.count * c.slices)), dim3(kThreads), 0, s, true, a, c, start, list, (int)in_vectors,
                          (int)out_vectors);
}

}  // namespace

cudaError_t launch_embed(int type, int param_type, const EmbedArgs &a, cudaStream_t s) {
    if (type == ZENO_F32) return param_type == ZENO_F32 ? embed<float, float>(a, s) : embed<float, __nv_bfloat16>(a, s);
    return param_type == ZENO_F32 ? embed<__nv_bfloat16, float>(a, s) : embed<__nv_bfloat16, __nv_bfloat16>(a, s);
}

int64_t embed_gradient_workspace(int m, int64_t n, int64_t vocab, int64_t cols) {
    const Classes c = classes_of(m, vocab, cols);
    return ((int64_t)m * c.count * c.starts() + m * n) * 4;
}

bool embed_gradient_fits(int m, int64_t vocab, int64_t cols) {
    const Classes c = classes_of(m, vocab, cols);
    return (int64_t)m * c.count * c.slices <= 0x7fffffff;
}

cudaError_t launch_embed_gradient(int type, int param_type, const EmbedGradArgs &a, cudaStream_t s) {
    if (type == ZENO_F32) return param_type == ZENO_F32 ? embed_gradient<float, float>(a, s) : embed_gradient<float, __nv_bfloat16>(a, s);
    return param_type == ZENO_F32 ? embed_gradient<__nv_bfloat16, float>(a, s) : embed_gradient<__nv_bfloat16, __nv_bfloat16>(a, s);
}

}  // namespace zeno

// Log probabilities of given tokens with entropy and top alternatives, and their gradient at the logits.
//
// Both directions are bound by the logits' bytes.  Forward: one pass with a running reference instead of the maximum, in
// powers of two: with t_j = z_j log2 e - M, S = sum 2^t_j and E = sum 2^t_j t_j for any M near the largest z log2 e,
//   lse = (M + log2 S) ln 2 (formed from M ln 2, rounded, and the remainder),   log p_j = (t_j - log2 S) ln 2,   entropy = (log2 S - E / S) ln 2;
// M moves by d: S' = 2^-d S, E' = 2^-d (E - d S).  No subtraction of nearly equal numbers besides those of the definition.
#include "zeno_operators.h"

namespace zeno {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// exp is zero in binary32 below this: a logarithm under it may be taken as it, so that zero times it is zero
constexpr float kLogOfNothing = -200.f;
// Rows whose largest logit is between -kFar and kFar go by powers of two: M, rounded, is there off the largest z log2 e by at most 8, so that
// no 2^t overflows.  Entries below -kFar (masks) are kept at that, where they add nothing to such a row.  Other rows (masked
// throughout, or not finite) are summed by the definition.
constexpr float kFar = 134217728.f;
constexpr int kChain = 4096;       // terms of a sum that one chain of additions may have
constexpr float kUnset = -kFar * kLog2e;      // the reference of nothing
constexpr float kSlack = 4.f;      // how far (in logits) the reference may fall behind the largest logit before it moves
constexpr int kMaxTop = ZENO_MAX_TOP;
constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ float exp2_fast(float t) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}

// 16 bytes of logits
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int N = 4;
    static constexpr uint32_t kFill = 0xff800000u;      // minus infinity
    // largest entry; a NaN counts only among nothing else
    static __device__ __forceinline__ float most(uint4 v) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    // entries in pairs, at least -kFar each (a NaN stays)
    static __device__ __forceinline__ void entries(uint4 v, Two (&o)[N / 2]) {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("max.NaN.f32 %0, %1, %2;" : "=f"(f[i]) : "f"(__uint_as_float(u[i])), "f"(-kFar));
        o[0] = Two{f[0], f[1]};
        o[1] = Two{f[2], f[3]};
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    static constexpr uint32_t kFill = 0xff80ff80u;
    static __device__ __forceinline__ __nv_bfloat162 pair(uint32_t u) { return *reinterpret_cast<__nv_bfloat162 *>(&u); }
    static __device__ __forceinline__ float most(uint4 v) {
        const __nv_bfloat162 m = __hmax2(__hmax2(pair(v.x), pair(v.y)), __hmax2(pair(v.z), pair(v.w)));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static __device__ __forceinline__ void entries(uint4 v, Two (&o)[N / 2]) {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
        const __nv_bfloat162 low = __float2bfloat162_rn(-kFar);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 m = __hmax2_nan(pair(u[i]), low);
            const uint32_t w = *reinterpret_cast<const uint32_t *>(&m);
            o[i] = Two{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
        }
    }
};

// Entries before the first 16-byte boundary of a row (all of a short one)
template <typename T>
__device__ __forceinline__ int64_t head_of(const T *p, int64_t count) {
    const int64_t h = (int64_t)((16u - (unsigned)(reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / (int64_t)sizeof(T);
    return h < count ? h : count;
}

struct Sums {
    float M, s, e;
    // to the reference `to`, not below M unless nothing has been added
    __device__ __forceinline__ void move(float to) {
        const float d = to - M, f = s == 0.f ? 0.f : exp2_fast(-d);
        e = f == 0.f ? 0.f : f * (e - d * s);
        s *= f;
        M = to;
    }
    __device__ __forceinline__ void add(float z) {
        const float t = fmaf(z, kLog2e, -M), p = exp2_fast(t);
        s += p;
        e = fmaf(p, t, e);
    }
};

// the sums of the first COUNT lanes (a power of two), in those
template <int COUNT>
__device__ __forceinline__ Sums join_first(Sums w) {
    float M = w.M;
#pragma unroll
    for (int k = COUNT / 2; k >= 1; k >>= 1) M = fmaxf(M, __shfl_xor_sync(kAll, M, k));
    w.move(M);
#pragma unroll
    for (int k = COUNT / 2; k >= 1; k >>= 1) {
        w.s += __shfl_xor_sync(kAll, w.s, k);
        w.e += __shfl_xor_sync(kAll, w.e, k);
    }
    return w;
}

// The unsigned half of rank_key: the order of the values, NaN with minus infinity
__device__ __forceinline__ uint32_t order_of(float z) { return (uint32_t)(rank_key(z, 0) >> 32); }
__device__ __forceinline__ float value_of_order(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }

// A warp's list of the largest keys, the k-th one in lane k - 1 (zero: none yet), and the value that a candidate has to reach.
struct TopList {
    unsigned long long mine = 0;
    uint32_t need = 0;
    // every candidate of the warp that is better than the last of `top`
    __device__ __forceinline__ void offer(unsigned long long key, int top, int lane) {
        unsigned todo = __ballot_sync(kAll, key > __shfl_sync(kAll, mine, top - 1));
        while (todo) {
            const int from = __ffs(todo) - 1;
            todo &= todo - 1;
            const unsigned long long k = __shfl_sync(kAll, key, from);
            const unsigned long long before = __shfl_up_sync(kAll, mine, 1);
            const bool later = k > mine;                              // this lane's entry moves back by one
            const bool first = lane == 0 || !(k > before);            // the new one's place, if it is before this entry
            if (later) mine = first ? k : before;
        }
        need = max(need, (uint32_t)(__shfl_sync(kAll, mine, top - 1) >> 32));
    }
};

// The row's sums by the definition, for a block: m (the largest entry, 0 for a row of minus infinities), sum exp(z - m) and the
// sum of those times z - m.
template <typename T, int THREADS>
__device__ __noinline__ void sums_by_definition(const T *z, int64_t vocab, float *scratch, float &m, float &s, float &e) {
    m = -INFINITY;
    for (int64_t j = threadIdx.x; j < vocab; j += THREADS) m = fmaxf(m, value_of(z + j));
#pragma unroll
    for (int k = 16; k >= 1; k >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, k));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = m;
    __syncthreads();
    for (int k = 0; k < THREADS / 32; ++k) m = fmaxf(m, scratch[k]);
    if (m == -INFINITY) m = 0.f;
    LongSum all_s, all_e;
    for (int64_t j = threadIdx.x; j < vocab;) {
        const int64_t end = min(vocab, j + kShortSum * THREADS);
        s = e = 0.f;
        for (; j < end; j += THREADS) {
            const float d = value_of(z + j) - m, p = exp2f(d * kLog2e);
            s += p;
            e = fmaf(p, fmaxf(d, kLogOfNothing), e);
        }
        all_s.add(s);
        all_e.add(e);
    }
    __syncthreads();
    s = block_sum<THREADS>(all_s.sum, scratch);
    __syncthreads();
    e = block_sum<THREADS>(all_e.sum, scratch);
}

// Places the better of `count` keys, which differ but for zeros (none), in their order: a key's place is the number of better ones.
template <int THREADS>
__device__ __forceinline__ void rank_keys(const unsigned long long *keys, int count, int top, unsigned long long *best) {
    for (int i = threadIdx.x; i < count; i += THREADS) {
        const unsigned long long k = keys[i];
        int place = 0;
        for (int c = 0; c < count; ++c) place += keys[c] > k;
        if (k && place < top) best[place] = k;
    }
}

// The best `top` of a stretch of vectors and the entries beside them, by lists that the warps keep: for rows in which too many
// entries reach what is known to be needed (ties above all).
template <typename T, int THREADS>
__device__ __noinline__ void top_by_lists(const T *z, int64_t head, int64_t v_begin, int64_t v_end, int64_t rest, int64_t rest_at, int top, uint32_t need,
                                          unsigned long long *keys, unsigned long long *best) {
    using V = Vec<T>;
    constexpr int kWarps = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    TopList list;
    list.need = need;
    for (int64_t base = v_begin + warp * 32; base < v_end; base += THREADS) {
        uint32_t u = 0;
        if (base + lane < v_end) u = order_of(V::most(reinterpret_cast<const uint4 *>(z + head)[base + lane]));
        // four lanes' vectors at a time (or eight), an entry to a lane
        constexpr int kSide = 32 / V::N;
        unsigned todo = __ballot_sync(kAll, u >= list.need);
        while (todo) {
            int from = -1;
            unsigned left = todo;
#pragma unroll
            for (int s = 0; s < kSide; ++s) {
                const int f = __ffs(left) - 1;
                left &= left - 1;
                if (lane / V::N == s) from = f;
            }
            todo = left;
            unsigned long long key = 0;
            if (from >= 0) {
                const int64_t j = head + (base + from) * V::N + lane % V::N;
                if (base + from < v_end) key = rank_key(value_of(z + j), (int)j);
            }
            list.offer(key, top, lane);
        }
    }
    if (warp == 0) {
        const int64_t j = lane < head ? lane : rest_at + lane;
        list.offer(lane < rest ? rank_key(value_of(z + j), (int)j) : 0, top, lane);
    }
    __syncthreads();
    if (lane < top) keys[warp * top + lane] = list.mine;
    __syncthreads();
    rank_keys<THREADS>(keys, kWarps * top, top, best);
}

// A row goes to a block, or (few rows) to a cluster of `parts` blocks that join through distributed shared memory.  A warp takes 32
// x kBatch vectors at a time, all loads ahead of their use.
//
// The alternatives cost the pass over the logits a comparison or two a batch: a thread keeps its largest entry, the batch it was in, and the largest
// of its other batches.  The k-th largest of the threads' largest is a bound that k entries reach, and only about k threads have
// entries that do, nearly always in one batch; those are read again, and what reaches the bound is ranked by counting.  (4096 x 131,072 bfloat16:
// 174 us without alternatives, 6.2 TB/s; 188 with four, 205 with 32; with lists kept by the warps during the pass 340 and 1,047, and with all of
// those threads' entries read again, by then from memory, 203 and 281.  8192 x 8000: 51 us, the row's end as long as the row.)
template <typename T, int THREADS, bool TOP>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 6 : THREADS == 128 ? 12 : 32) logprobs_kernel(LogprobArgs a, int parts) {
    using V = Vec<T>;
    constexpr int kWarps = THREADS / 32, kBatch = 4, kMaxParts = 8, kKeys = 512;
    static_assert(kKeys >= kWarps * kMaxTop && kKeys >= kMaxParts * kMaxTop, "the lists of all warps, of all parts");
    __shared__ float scratch[kWarps];
    __shared__ float warp_sums[kWarps][3];
    __shared__ float sums[3];
    __shared__ unsigned long long keys[TOP ? kKeys : 1];
    __shared__ unsigned long long best[TOP ? kMaxTop : 1];
    __shared__ uint32_t orders[TOP ? THREADS : 1];     // the threads' largest entries
    __shared__ uint16_t hits[TOP ? THREADS : 1];       // the threads to look at again
    __shared__ uint32_t bound;
    __shared__ int hit_batch[TOP ? THREADS : 1];
    __shared__ int n_single, n_whole, n_keys;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t r = (int)(blockIdx.x / (unsigned)parts);
    const int part = (int)(blockIdx.x - (unsigned)r * (unsigned)parts);
    const T *z = static_cast<const T *>(a.logits.data) + a.logits.at(r);
    const int top = a.top;

    const int target = a.logprobs && threadIdx.x == 0 && part == 0 ? a.targets[r] : -1;     // its logit is asked for when this has come
    const int64_t head = head_of(z, a.vocab), vecs = (a.vocab - head) / V::N;
    const int64_t v_begin = vecs * part / parts, v_end = vecs * (part + 1) / parts;
    const uint4 *zv = reinterpret_cast<const uint4 *>(z + head);
    // Until an entry is above -kFar the reference M is 0, where all others (kept at least -kFar) add nothing.
    float limit = -kFar;                               // the reference moves for entries beyond this
    float largest = -INFINITY, second = -INFINITY;     // of the batches' largest entries; and which batch's
    int batch = 0, largest_batch = 0;
    float M = 0.f;
    Two s2 = both(0.f), e2 = both(0.f);
    auto move = [&](float to) {
        Sums p = {M, s2.x, e2.x}, q = {M, s2.y, e2.y};
        p.move(to);
        q.move(to);
        s2 = Two{p.s, q.s};
        e2 = Two{p.e, q.e};
        M = to;
    };
    bool any = false;

    for (int64_t base = v_begin + warp * 32 * kBatch; base < v_end; base += THREADS * kBatch) {
        uint4 raw[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int64_t v = base + i * 32 + lane;
            raw[i] = v < v_end ? __ldcs(zv + v) : make_uint4(V::kFill, V::kFill, V::kFill, V::kFill);
            any |= v < v_end;
        }
        float most = V::most(raw[0]);
#pragma unroll
        for (int i = 1; i < kBatch; ++i) most = fmaxf(most, V::most(raw[i]));
        if (TOP) {
            if (most > largest) {
                second = largest;
                largest = most;
                largest_batch = batch;
            } else {
                second = fmaxf(second, most);
            }
            ++batch;
        }
        if (most > limit) {
            move(__fmul_rn(most, kLog2e));       // rounded before it is subtracted from anything
            limit = most + kSlack;
        }
        const Two c = both(kLog2e), m = both(-M);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            Two f[V::N / 2];
            V::entries(raw[i], f);
#pragma unroll
            for (int k = 0; k < V::N / 2; ++k) {
                const Two t = fma2(f[k], c, m), p = {exp2_fast(t.x), exp2_fast(t.y)};
                s2 = add2(s2, p);
                e2 = fma2(p, t, e2);
            }
        }
    }
    const bool given = target >= 0 && target < a.vocab;
    const float zt = given ? value_of(z + target) : 0.f;
    // what lies before the first vector and behind the last: fewer than 2 N entries
    const int64_t rest = part == 0 ? a.vocab - vecs * V::N : 0, rest_at = vecs * V::N;
    const int64_t rest_j = lane < head ? lane : rest_at + lane;
    const bool has_rest = warp == 0 && lane < rest;
    const float v_rest = has_rest ? value_of(z + rest_j) : -INFINITY;
    if (has_rest) {
        if (v_rest > limit) {
            move(__fmul_rn(v_rest, kLog2e));
            limit = v_rest;
        }
        Sums p = {M, s2.x, e2.x};
        p.add(v_rest < -kFar ? -kFar : v_rest);
        s2.x = p.s;
        e2.x = p.e;
        any = true;
    }
    // The warps' sums and the threads' largest entries; then one warp joins the sums, and another finds the bound: what the largest entries of
    // `top` threads and few more reach.
    Sums q = {limit == -kFar ? kUnset : M, s2.x + s2.y, e2.x + e2.y};
    q = join_first<32>(q);
    if (lane == 0) {
        warp_sums[warp][0] = q.M;
        warp_sums[warp][1] = q.s;
        warp_sums[warp][2] = q.e;
    }
    if (TOP) {
        orders[threadIdx.x] = any ? order_of(fmaxf(largest, v_rest)) : 0u;
        if (threadIdx.x == 0) n_single = n_whole = n_keys = 0;
    }
    __syncthreads();
    if (warp == kWarps - 1) {
        Sums w = {kUnset, 0.f, 0.f};
        if (lane < kWarps) w = {warp_sums[lane][0], warp_sums[lane][1], warp_sums[lane][2]};
        w = join_first<kWarps>(w);
        if (lane == 0) {
            sums[0] = w.M;
            sums[1] = w.s;
            sums[2] = w.e;
        }
    }
    if (TOP && warp == 0) {
        uint32_t o[kWarps], at_least = 0;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) o[k] = orders[k * 32 + lane];
        uint32_t lowest = ~0u, highest = 0;
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
            lowest = min(lowest, o[k]);
            highest = max(highest, o[k]);
        }
        // `top` threads and more reach at_least, fewer than `top` reach beyond; a few more than wanted will do
        at_least = __reduce_min_sync(kAll, lowest);
        uint32_t beyond = __reduce_max_sync(kAll, highest);
        if (at_least < beyond) {
            ++beyond;
            while (beyond - at_least > 1) {
                const uint32_t next = at_least + (beyond - at_least) / 2;
                int n = 0;
#pragma unroll
                for (int k = 0; k < kWarps; ++k) n += o[k] >= next;
                n = (int)__reduce_add_sync(kAll, (unsigned)n);
                if (n < top) beyond = next;
                else at_least = next;
                if (n >= top && n <= top + 8) break;
            }
        }
        if (lane == 0) bound = at_least;
    }
    __syncthreads();
    if (TOP) {
        const uint32_t need = bound, own = orders[threadIdx.x];
        if (own >= need && any) {         // from the front: one batch to read again; from the back: all of them
            if (order_of(second) >= need) {
                hits[THREADS - 1 - atomicAdd(&n_whole, 1)] = (uint16_t)threadIdx.x;
            } else {
                const int at = atomicAdd(&n_single, 1);
                hits[at] = (uint16_t)threadIdx.x;
                hit_batch[at] = largest_batch;
            }
        }
        auto offer = [&](float v, int64_t j) {
            if (order_of(v) < need) return;
            const int at = atomicAdd(&n_keys, 1);
            if (at < kKeys) keys[at] = rank_key(v, (int)j);
        };
        if (has_rest) offer(v_rest, rest_j);
        __syncthreads();
        const int per = (int)((v_end - v_begin + THREADS * kBatch - 1) / (THREADS * kBatch)) * kBatch;        // a thread's vectors
        const int singles = n_single * kBatch, vectors = singles + n_whole * per;
        const bool few = n_single + n_whole <= 2 * top + 32;
        if (few) {
            constexpr int kAtOnce = 4;                // loads in flight
            for (int i0 = threadIdx.x; i0 < vectors; i0 += THREADS * kAtOnce) {
                uint4 raw[kAtOnce];
                int64_t at[kAtOnce];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int i = i0 + u * THREADS;
                    at[u] = v_end;
                    if (i < vectors) {
                        const int k = i < singles ? hit_batch[i / kBatch] * kBatch + i % kBatch : (i - singles) % per;
                        const int who = hits[i < singles ? i / kBatch : THREADS - 1 - (i - singles) / per];
                        at[u] = v_begin + (int64_t)(k / kBatch) * THREADS * kBatch + (who >> 5) * 32 * kBatch + k % kBatch * 32 + (who & 31);
                    }
                    if (at[u] < v_end) raw[u] = __ldcg(zv + at[u]);
                }
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u)
                    if (at[u] < v_end && order_of(V::most(raw[u])) >= need) {
                        T e[V::N];
                        *reinterpret_cast<uint4 *>(e) = raw[u];
#pragma unroll
                        for (int n = 0; n < V::N; ++n) offer(value_of(e + n), head + at[u] * V::N + n);
                    }
            }
        }
        __syncthreads();
        if (few && n_keys <= kKeys) rank_keys<THREADS>(keys, n_keys, top, best);
        else top_by_lists<T, THREADS>(z, head, v_begin, v_end, rest, rest_at, top, need, keys, best);
        __syncthreads();
    }

    if (parts > 1) {
        cluster_barrier();
        if (part == 0) {
            if (warp == 0) {
                Sums w = {kUnset, 0.f, 0.f};
                if (lane < parts) {
                    w.M = cluster_load(cluster_addr(&sums[0], lane));
                    w.s = cluster_load(cluster_addr(&sums[1], lane));
                    w.e = cluster_load(cluster_addr(&sums[2], lane));
                }
                w = join_first<kMaxParts>(w);
                __syncwarp();                                  // lane 0's loads are from here too
                if (lane == 0) {
                    sums[0] = w.M;
                    sums[1] = w.s;
                    sums[2] = w.e;
                }
            }
            if (TOP) {
                for (int i = threadIdx.x; i < parts * top; i += THREADS) keys[i] = cluster_load64(cluster_addr(&best[i % top], i / top));
                __syncthreads();
                rank_keys<THREADS>(keys, parts * top, top, best);
            }
        }
        cluster_barrier();
        if (part != 0) return;
    }
    q = {sums[0], sums[1], sums[2]};

    const bool plain = a.long_sums || !(fabsf(q.M) <= 0.99f * kFar * kLog2e);
    float m, log_s, mean_t;
    if (plain) {
        float s, e;
        sums_by_definition<T, THREADS>(z, a.vocab, scratch, m, s, e);
        log_s = logf(s);
        mean_t = s == 0.f ? log_s : e / s;                // a row of nothing: entropy 0
    } else {
        m = q.M;
        log_s = log2f(q.s);
        mean_t = q.e / q.s;
    }
    auto log_prob = [&](float v) {
        if (plain) return log_s == -INFINITY ? -INFINITY : (v - m) - log_s;
        if (v < -kFar) return v - (m + log_s) * kLn2;     // its product with log2 e may be beyond binary32
        const float lp = (fmaf(v, kLog2e, -m) - log_s) * kLn2;
        return lp > 0.f ? 0.f : lp;                       // a rounding above the definition's bound
    };
    if (threadIdx.x == 0) {
        if (a.lse) {
            // M / log2 e as a logit: what its rounding is off by joins log2 S, and only the last addition rounds at the size of lse
            const float at = m * kLn2;
            a.lse[r] = plain ? m + log_s : at + (log_s - fmaf(at, kLog2e, -m)) * kLn2;
        }
        if (a.entropy) {
            const float h = log_s == -INFINITY ? 0.f : (log_s - mean_t) * (plain ? 1.f : kLn2);
            a.entropy[r] = h < 0.f ? 0.f : h;             // a rounding under the definition's bound
        }
        if (a.logprobs) a.logprobs[r] = given ? log_prob(zt) : 0.f;
    }
    if (TOP && (int)threadIdx.x < top) {
        const unsigned long long key = best[threadIdx.x];
        if (a.top_idx) a.top_idx[r * top + threadIdx.x] = (int)(0xffffffffu - (uint32_t)key);
        if (a.top_logprobs) a.top_logprobs[r * top + threadIdx.x] = log_prob(value_of_order((uint32_t)(key >> 32)));
    }
}

// The gradient: bound by reading and writing each logit once (4096 x 65,536 bfloat16: 160 us, 6.7 TB/s).
// Elements in a block of its kernel: two rounds of four vectors a thread, half of them in flight.
constexpr int kGradThreads = 256, kGradBatch = 4;

// An lse in binary32 is off by half a step, and so relative to them are all of a row's probabilities.  From 2^8 on (binary32, 2^-17 below; 2^12 and
// 2^-13 for a gradient in bfloat16, whose own half step is 2^-9) that is more than the rest of the arithmetic: the row is summed again, by the block
// that then does all of it, since the gradient may lie over the logits (4096 x 65,536 binary32: 501 us, 322 near zero; 61 x 50,001: 27 and 12).
template <typename T> constexpr float kFarLse = sizeof(T) == 4 ? 256.f : 4096.f;

// Sum of exp(z - lse) over a row, for a block: what a rounded lse leaves to be taken off every log probability.  Near 1 as far as lse is right.
template <typename T>
__device__ __noinline__ float sum_beside(const T *z, int64_t vocab, float lse, float *scratch) {
    using V = Vec<T>;
    const int64_t head = head_of(z, vocab), vecs = (vocab - head) / V::N, rest = vocab - vecs * V::N;
    const uint4 *zv = reinterpret_cast<const uint4 *>(z + head);
    LongSum s;
    if (threadIdx.x < rest) s.sum = exp2_fast((value_of(z + (threadIdx.x < head ? threadIdx.x : vecs * V::N + threadIdx.x)) - lse) * kLog2e);
    for (int64_t base = threadIdx.x; base < vecs; base += kGradThreads * kGradBatch) {
        uint4 raw[kGradBatch];
#pragma unroll
        for (int i = 0; i < kGradBatch; ++i) raw[i] = base + i * kGradThreads < vecs ? zv[base + i * kGradThreads] : make_uint4(V::kFill, V::kFill, V::kFill, V::kFill);
        float part = 0.f;
#pragma unroll
        for (int i = 0; i < kGradBatch; ++i) {
            T e[V::N];
            *reinterpret_cast<uint4 *>(e) = raw[i];
#pragma unroll
            for (int k = 0; k < V::N; ++k) part += exp2_fast((value_of(e + k) - lse) * kLog2e);
        }
        s.add(part);
    }
    return block_sum<kGradThreads>(s.sum, scratch);
}

// One element: what the row's sums say and the upstream gradients ask for; the target's own term is added apart.  `beside`: log of the above.
template <bool ENTROPY>
__device__ __forceinline__ float token_slope(float z, float lse, float beside, float g, float h, float entropy) {
    const float lp = (z - lse) - beside, p = exp2_fast(lp * kLog2e);
    return -p * (ENTROPY ? fmaf(h, fmaxf(lp, kLogOfNothing) + entropy, g) : g);
}

// A block takes `chunk` entries of a row, in vectors that are aligned in the gradient.  VECTORS: and in the logits, where they are put together from
// the two that they lie in otherwise (1024 x 65,536 of rows 3 longer, bfloat16: 50 us; 45 where they are aligned, 141 by single entries).
template <typename T, bool ENTROPY, bool VECTORS>
__global__ void __launch_bounds__(kGradThreads) token_gradient_kernel(TokenGradArgs a, unsigned chunks, int64_t chunk) {
    using V = Vec<T>;
    const int64_t r = (int)(blockIdx.x / chunks);
    const int64_t first = (int64_t)(blockIdx.x - (unsigned)r * chunks) * chunk;
    const T *z = static_cast<const T *>(a.logits.data) + a.logits.at(r);
    T *out = static_cast<T *>(a.grad.data) + a.grad.at(r);
    const int t = a.targets[r];
    const bool given = t >= 0 && t < a.vocab;
    const float lse = a.lse[r], g = given ? a.g_logprob[r] : 0.f, h = ENTROPY ? a.g_entropy[r] : 0.f, entropy = ENTROPY ? a.entropy[r] : 0.f;
    const bool zero = (!given && !ENTROPY) || lse == -INFINITY;
    float beside = 0.f;
    int64_t last = first + chunk;
    if (!zero && fabsf(lse) >= kFarLse<T>) {       // one block for the row, which it reads as a whole before it writes: the gradient may lie there
        if (first != 0) return;
        __shared__ float scratch[kGradThreads / 32];
        beside = logf(sum_beside(z, a.vocab, lse, scratch));
        last = a.vocab;
    }
    auto one = [&](int64_t j) {
        float v = 0.f;
        if (!zero) v = token_slope<ENTROPY>(value_of(z + j), lse, beside, g, h, entropy) + (j == t && given ? g : 0.f);
        put(out + j, v);
    };
    // the vectors from v_first to v_end; what lies before and behind, at most 4 N entries, by single ones.  Of the first and last vector of a row whose
    // logits lie otherwise one half would come from outside of it.
    const int64_t head = head_of(out, a.vocab), vecs = (a.vocab - head) / V::N;
    const int64_t v_first = VECTORS ? 0 : min(vecs, (int64_t)1), v_end = VECTORS ? vecs : max(v_first, vecs - 1);
    const int64_t before = head + v_first * V::N;
    if (first == 0 && threadIdx.x < a.vocab - (v_end - v_first) * V::N)
        one(threadIdx.x < before ? threadIdx.x : (v_end - v_first) * V::N + threadIdx.x);
    const unsigned off = (unsigned)(reinterpret_cast<uintptr_t>(z + head) & 15);
    const uint4 *zv = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(z + head) - off);
    uint4 *ov = reinterpret_cast<uint4 *>(out + head);
    const int64_t end = min((last + V::N - 1) / V::N, v_end);
    for (int64_t base = max(first / V::N, v_first) + threadIdx.x; base < end; base += kGradThreads * kGradBatch) {
        uint4 raw[kGradBatch], more[VECTORS ? 1 : kGradBatch];
        if (!zero)
#pragma unroll
            for (int i = 0; i < kGradBatch; ++i)
                if (base + i * kGradThreads < end) {
                    raw[i] = zv[base + i * kGradThreads];
                    if (!VECTORS) more[i] = zv[base + i * kGradThreads + 1];
                }
#pragma unroll
        for (int i = 0; i < kGradBatch; ++i) {
            const int64_t v = base + i * kGradThreads;
            if (v >= end) break;
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if (!zero) {
                T e[V::N], o[V::N];
                *reinterpret_cast<uint4 *>(e) = VECTORS ? raw[i] : shifted<sizeof(T)>(raw[i], more[VECTORS ? 0 : i], off);
                const int64_t at = (int64_t)t - (head + v * V::N);
#pragma unroll
                for (int k = 0; k < V::N; ++k) {
                    float s = token_slope<ENTROPY>(value_of(e + k), lse, beside, g, h, entropy);
                    if (at == k) s += g;                       // g is 0 without a target
                    put(o + k, s);
                }
                w = *reinterpret_cast<uint4 *>(o);
            }
            ov[v] = w;
        }
    }
}

template <typename T, int THREADS>
cudaError_t launch_logprobs(LogprobArgs a, int parts, cudaStream_t s) {
    a.long_sums = a.vocab > (int64_t)kChain * THREADS * 2 * parts;       // more than kChain terms to each of a thread's sums
    auto *kernel = a.top ? logprobs_kernel<T, THREADS, true> : logprobs_kernel<T, THREADS, false>;
    const dim3 grid((unsigned)(a.m * a.n * parts));
    return parts > 1 ? launch_clustered(kernel, parts, grid, dim3(THREADS), 0, s, false, a, parts) : launch_chained(kernel, grid, dim3(THREADS), 0, s, false, a, parts);
}

// Threads to a row, and blocks.  A warp alone has no barriers between its sums, the bound and the alternatives: 8192 x 1000 bfloat16 12 us, with eight
// alternatives 21 (128 threads: 21, 37), binary32 14, 23 (21, 39); 3003 x 3279 12, 19 (14, 21); few rows are even (200 x 2000 8, 12; 6, 10).  Not so with 32
// alternatives, where every lane reaches the bound and nearly all of the row is read again: 3003 x 3279 70 us, 25 with 128 threads; 8192 x 1000
// 74, but 320 there (fewer vectors than threads, so that lists are kept).  128 threads against 256, none / eight / 32 alternatives: 4096 x 8000 bfloat16
// 23 / 31 / 37 and 27 / 39 / 45, binary32 31 / 45 / 53 and 31 / 51 / 57; 2000 x 16,000 21 / 27 / 31 and 23 / 29 / 33, 33 / 45 / 51 and 31 / 45 / 47.
// Rows are cut until there are two blocks an SM.  Up to what is resident (888 blocks) 200 x 70,208 binary32 takes 18 / 25 / 27 us and not
// 23 / 33 / 35, 102 x 39,744 with 32 alternatives 27 and not 18, 150 x 32,000 bfloat16 with eight 14 and not 12.
template <typename T>
cudaError_t token_logprobs(const LogprobArgs &a, cudaStream_t s) {
    const int64_t rows = a.m * a.n;
    if (a.vocab <= 2048 || (a.vocab <= 4096 && rows >= 16 * 148)) return launch_logprobs<T, 32>(a, 1, s);
    if (a.vocab <= 16384 && rows >= 148) return launch_logprobs<T, 128>(a, 1, s);
    int parts = 8;
    while (parts > 1 && (rows * parts > 296 || a.vocab < parts * 2048)) parts /= 2;
    return launch_logprobs<T, 256>(a, parts, s);
}

template <typename T>
cudaError_t token_gradient(const TokenGradArgs &a, cudaStream_t s) {
    const int64_t rows = a.m * a.n;
    int64_t chunk = 2 * kGradBatch * kGradThreads * Vec<T>::N;
    while (rows * ((a.vocab + chunk - 1) / chunk) > 0x7fffffff) chunk *= 2;
    const unsigned chunks = (unsigned)((a.vocab + chunk - 1) / chunk);
    // every row of both at the same offset from a 16-byte boundary
    const bool vectors = ((reinterpret_cast<uintptr_t>(a.logits.data) - reinterpret_cast<uintptr_t>(a.grad.data)) & 15) == 0 &&
                         (a.n <= 1 || (a.logits.row - a.grad.row) * (int64_t)sizeof(T) % 16 == 0) &&
                         (a.m <= 1 || (a.logits.group - a.grad.group) * (int64_t)sizeof(T) % 16 == 0);
    auto *kernel = a.g_entropy ? (vectors ? token_gradient_kernel<T, true, true> : token_gradient_kernel<T, true, false>)
                               : (vectors ? token_gradient_kernel<T, false, true> : token_gradient_kernel<T, false, false>);
    return launch_chained(kernel, dim3((unsigned)(rows * chunks)), dim3(kGradThreads), 0, s, false, a, chunks, chunk);
}

}  // namespace

cudaError_t launch_token_logprobs(int type, const LogprobArgs &a, cudaStream_t s) {
    return type == ZENO_BF16 ? token_logprobs<__nv_bfloat16>(a, s) : token_logprobs<float>(a, s);
}

cudaError_t launch_token_gradient(int type, const TokenGradArgs &a, cudaStream_t s) {
    return type == ZENO_BF16 ? token_gradient<__nv_bfloat16>(a, s) : token_gradient<float>(a, s);
}

}  // namespace zeno

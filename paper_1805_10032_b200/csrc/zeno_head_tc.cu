// The products around the output layer on the tensor cores: logits with the sums of their exponentials, the probabilities' gradient from
// logits computed again, and its two products.
//
// A pair of blocks (a cluster of two SMs; a single one, with a tile of 128 rows, for the logits of groups that have no more) takes a tile of 256 rows by 256 or
// 128 columns: the pair's instruction (cta_group::2, M = 256) reads 128 rows of A and half of the columns of B from each block's shared memory, so that a block copies half of what the tile needs, and leaves 128 rows of sums in either
// block's TMEM.  Operands are bfloat16, in binary32 sums; a binary32 operand is three terms whose products are summed one pair of terms after the other, the
// leading pair last.  X and W lie with the contraction's index contiguous for the logits ("K-major"); P W takes W, and P^T X both, with the index of the
// result contiguous ("MN-major"), all in the 128-byte swizzled layouts that the tensor copies write.
//   warp 0: copies, both blocks' counted on the first one's barriers;  warp 1 of the first block: the pair's instructions;
//   the other warps: sums from TMEM, the next tile's being formed meanwhile: 32 rows and 64 or 128 columns each.
// One lane each loops over the copies and the instructions: by whole warps that elect a lane for every stage, a stage takes 500 cycles whatever its size
// (256 by 128 tiles: 400), and with the second block's copies counted on its own barriers and reported to the first, 580.
#include "zeno_head.h"
#include "zeno_tc.cuh"

namespace zeno {

namespace {

constexpr int kBlockRows = 128;                     // rows of a tile that a block has
constexpr int kK = 64;                               // contraction indices of a stage: 128 bytes
constexpr int kABytes = kBlockRows * kK * 2;
constexpr int kBox = 4096;                           // 32 rows of 128 bytes of a warp on their way out
constexpr int kBoundsKept = 48;                      // groups whose bounds are kept in shared memory

template <HeadStep STEP, int N, int COLS, int BLOCKS>
struct Shape {
    static constexpr int kHalf = N / BLOCKS;                             // of the columns, in a block
    static constexpr int kRows = BLOCKS * kBlockRows;
    static constexpr int kBBytes = kHalf * kK * 2;
    static constexpr int kStageBytes = kABytes + kBBytes;
    static constexpr int kCols = COLS;                                   // of a warp that takes sums
    static constexpr int kEpiWarps = 4 * N / kCols, kThreads = 32 * (2 + kEpiWarps);
    static constexpr int kBoxes = STEP == HeadStep::kSums ? 0 : STEP == HeadStep::kWeights ? 2 : 1;      // of a warp
    static constexpr int kBoxBytes = kEpiWarps * kBoxes * kBox;
    static constexpr int kStages = (225 * 1024 - kBoxBytes) / kStageBytes;
    static constexpr int kSmem = kStages * kStageBytes + kBoxBytes + 1024;
};

__device__ unsigned g_given_up;                      // blocks whose bounded waits gave up since the process began

// The tensor core adds with truncation towards zero, about 1.4e-8 of a sum with every 16 products (where all are positive).  So a set of sums in TMEM takes a
// stretch of the contraction only, and goes on in registers, in additions to nearest.  Stretches of 256 where binary32 operands are multiplied (by 512,
// gradients are off by 1.3 times as much as by plain products in binary32), of 128 for their logits, whose error a probability near one multiplies (3 x 57 tokens, 5001
// words by 777 columns: dx off by 4.4e-7, dW by 3.1e-7, by 256 by 7.5e-7 and 7.0e-7 in the same 96 us; 2048 tokens, 40576 words by 4096 9.7 ms, by 256 9.2); of 512
// for logits of bfloat16 operands (4096 tokens, 131072 words by 4096 columns: 2.83 ms, by 256 2.94, by 128 3.28; lse of 32768 of the words off by 1.9e-7, 0.9e-7,
// 0.5e-7, by plain products in binary32 0.6e-7), for D's as for lse's, so that a row's probabilities are those that lse is the sum of; of 1,024 for gradients that
// are rounded to bfloat16 anyway.
// The terms' planes of a stretch stay in L2 for all pairs of terms.
constexpr int kDrainTerms = 4, kDrainLogits = 2, kDrain = 8, kDrainBf16 = 16;

struct KernelArgs {
    HeadTcArgs h;
    int row_tiles, col_tiles;                        // row_tiles: at most, of a group
    int drain;                                       // blocks of kK contraction indices of a stretch
    int manual_stores;                               // kWeights: rows that no tensor copy can write
    uint32_t spin_limit;
};

__device__ __forceinline__ void remote_arrive(uint32_t addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
// an arrival on the barrier at this place in all of a tile's blocks, once the instructions so far have ended
template <int BLOCKS>
__device__ __forceinline__ void commit_to_all(uint32_t bar) {
    if constexpr (BLOCKS == 1) tc_commit(bar);
    else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
template <int BLOCKS>
__device__ __forceinline__ void mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    if constexpr (BLOCKS == 1)
        asm volatile(
            "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile(
            "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n"
            ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// MN-major operand: rows of 64 contiguous entries, one for each value of the contraction index; eight of them make a group of 1024 bytes, the next 64
// entries lie kK rows on.
__device__ __forceinline__ uint64_t mn_major(uint32_t addr) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3ffffu) >> 4);
    d |= (uint64_t)((kK * 128) >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
// A copy into this block's shared memory whose bytes are counted on a barrier of the tile's first block.
template <int BLOCKS>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, uint32_t bar) {
    if constexpr (BLOCKS == 1)
        tma_load_3d(dst, map, c0, c1, c2, bar);
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
            ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}
__device__ __forceinline__ void store_box(const CUtensorMap *map, const void *smem, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(smem_u32(smem)), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void add_box(const CUtensorMap *map, const void *smem, int c0, int c1, int c2) {
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(smem_u32(smem)), "r"(c0), "r"(c1), "r"(c2)
                 : "memory");
}
__device__ __forceinline__ void boxes_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void boxes_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT < 0 ? 0 : LEFT) : "memory");
}
__device__ __forceinline__ void boxes_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// What follows a narrow layer's logits takes two sums, or products, at a time, half the instructions (7168 tokens, 60000 words by 64 columns: 261 us, so 248).
__device__ __forceinline__ Two two_at(const float *f) { return Two{f[0], f[1]}; }
__device__ __forceinline__ void put_two(float *f, Two v) { f[0] = v.x, f[1] = v.y; }
constexpr float kLog2e = 1.4426950408889634f, kLog2eRest = (float)(1.4426950408889634 - (double)kLog2e);

// Division by the same number again and again: a multiplication by its reciprocal, rounded down, whose quotient is at most two too small.
struct Divisor {
    uint32_t d, m;
    __device__ explicit Divisor(uint32_t by) : d(by), m(0xffffffffu / by) {}
    __device__ __forceinline__ uint32_t operator()(uint32_t a) const {
        uint32_t q = __umulhi(a, m), rest = a - q * d;
        if (rest >= d) ++q, rest -= d;
        return rest >= d ? q + 1 : q;
    }
};

// head_tile() by reciprocals: of kHeadBand * col_tiles, and of the rows of the last band.  (Bound by the exponentials' unit, which divisions' conversions take
// turns on: 7168 tokens, 60000 words by 64 columns: 235 us, by divisions 248.)
__device__ __forceinline__ HeadTile head_tile(uint32_t t, uint32_t row_tiles, const Divisor &band_tiles, const Divisor &last_rows) {
    const uint32_t band = band_tiles(t), in = t - band * band_tiles.d;
    const bool whole = (band + 1) * kHeadBand <= row_tiles;
    const uint32_t col = whole ? in / kHeadBand : last_rows(in), rows = whole ? kHeadBand : last_rows.d;
    return HeadTile{(int)(band * kHeadBand + in - col * rows), (int)col};
}

// One tile and the part of the contraction that goes into it.
struct Item {
    int group, row0, rows_end, col0, k0, len, kb0, kb1, split, splits, extra;          // k0, len: the contraction's indices, kb0, kb1: blocks of kK of them
};

template <HeadStep STEP, int N, int COLS, int BLOCKS, typename P>
__global__ void __launch_bounds__((Shape<STEP, N, COLS, BLOCKS>::kThreads), 1) head_tc_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                              const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_extra, const KernelArgs args) {
    using S = Shape<STEP, N, COLS, BLOCKS>;
    constexpr int HN = S::kHalf, kCols = COLS;
    static_assert(BLOCKS == 2 || STEP == HeadStep::kSums || STEP == HeadStep::kProbs || STEP == HeadStep::kLogits, "few rows");
    constexpr bool kAMn = STEP == HeadStep::kWeights, kBMn = STEP == HeadStep::kWeights || STEP == HeadStep::kInputs;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    // full, empty [kStages]; dfull, dempty [2]
    constexpr int kBars = 2 * S::kStages + 4;
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ __align__(8) uint64_t drain_bar, never_bar;
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_state[kAbortWords];
    __shared__ uint32_t issued[2][S::kStages];                 // of each block (the first one knows both at the end): last round that copies were issued into a stage
                                                               // in, plus one, times four; whether they were of this block's rows (1), and of the other's (2)
    __shared__ int other_gave_up;
    __shared__ int bounds[2 * kBoundsKept];                    // begin and end of each group

    const HeadTcArgs &h = args.h;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = BLOCKS == 1 ? 0 : (int)cluster_rank();
    uint8_t *ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *boxes = ring + S::kStages * S::kStageBytes;
    auto full = [&](int s) { return smem_u32(&bars[s]); };
    auto empty = [&](int s) { return smem_u32(&bars[S::kStages + s]); };
    auto dfull = [&](int q) { return smem_u32(&bars[2 * S::kStages + q]); };
    auto dempty = [&](int q) { return smem_u32(&bars[2 * S::kStages + 2 + q]); };

    if (tid == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
    }
    if (tid == 0) {
        abort_state[0] = 0;
        abort_state[1] = (int)args.spin_limit;
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(full(s), 1);
            mbar_init(empty(s), 1);
            issued[0][s] = issued[1][s] = 0;
        }
        for (int q = 0; q < 2; ++q) {
            mbar_init(dfull(q), 1);
            mbar_init(dempty(q), BLOCKS * S::kEpiWarps);
        }
        mbar_init(smem_u32(&drain_bar), 1);
        mbar_init(smem_u32(&never_bar), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if constexpr (BLOCKS == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(2 * N) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(2 * N) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    tc_fence_before();
    __syncthreads();
    if (BLOCKS == 2) cluster_barrier();       // the other block's barriers are there
    tc_fence_after();
    pdl_wait();
    if (!h.last) pdl_launch_dependents();     // by a kernel of this call, never by the next call's
    const uint32_t tmem = tmem_base_slot;
    volatile int *abortp = &abort_state[0];

    const uint32_t pair = blockIdx.x / BLOCKS, pairs_of_blocks = gridDim.x / BLOCKS;
    // The tiles in their order: rows first within a band of kBand tiles, then columns, so that pairs next to one another share the columns' operand and all
    // of a band's rows stay in L2.
    const bool in_smem = h.groups <= kBoundsKept;
    if (in_smem && tid < 2 * h.groups) bounds[tid] = __ldcg((tid & 1 ? h.end : h.begin) + (tid >> 1));
    __syncthreads();
    auto begin_of = [&](int group) { return in_smem ? bounds[2 * group] : __ldcg(h.begin + group); };
    auto end_of = [&](int group) { return in_smem ? bounds[2 * group + 1] : __ldcg(h.end + group); };
    const uint32_t row_tiles = STEP != HeadStep::kWeights && h.groups == 1 ? min(args.row_tiles, (bounds[1] + S::kRows - 1) / S::kRows) : args.row_tiles;
    const uint32_t per_group = row_tiles * args.col_tiles, tiles = per_group * h.groups;
    // kInputs: whole rounds of tiles, then the rest of them, cut along the words so that it takes all pairs
    const uint32_t whole = STEP == HeadStep::kInputs ? tiles / pairs_of_blocks * pairs_of_blocks : tiles;
    const int splits = STEP == HeadStep::kInputs ? head_splits(tiles, pairs_of_blocks, h.most_splits) : 1;
    const uint32_t items = STEP == HeadStep::kLogits ? tiles * h.logits_parts : whole + (tiles - whole) * splits;
    const Divisor group_tiles(max(per_group, 1u)), band_tiles(kHeadBand * args.col_tiles), last_rows(max(row_tiles % kHeadBand, 1u));
    // false: no further item
    auto get_item = [&](int li, Item &it) {
        const uint32_t item = pair + li * pairs_of_blocks;
        if (item >= items) return false;
        uint32_t tile = item;
        it.split = 0;
        it.splits = 1;
        if (STEP == HeadStep::kInputs && item >= whole) {
            tile = whole + (item - whole) / splits;
            it.split = (int)(item - whole - (tile - whole) * splits);
            it.splits = splits;
        }
        if (STEP == HeadStep::kLogits) {
            it.splits = h.logits_parts;
            tile = item / it.splits;
            it.split = (int)(item - tile * it.splits);
        }
        it.extra = (int)(item - whole);
        HeadTile at;
        if constexpr (STEP == HeadStep::kSums || STEP == HeadStep::kProbs) {
            it.group = (int)group_tiles(tile);
            at = head_tile(tile - it.group * per_group, row_tiles, band_tiles, last_rows);
        } else {                                                          // whose warps have no registers to spare
            it.group = (int)(tile / per_group);
            at = zeno::head_tile(tile - it.group * per_group, row_tiles, args.col_tiles);
        }
        it.col0 = at.col * N;
        if (STEP == HeadStep::kWeights) {
            it.row0 = at.row * S::kRows;                                 // words of the piece
            it.rows_end = (int)h.piece;
            it.k0 = begin_of(it.group);
            it.len = end_of(it.group) - it.k0;
            it.kb0 = 0;
            it.kb1 = (it.len + kK - 1) / kK;
        } else {
            it.k0 = 0;
            it.len = (int)(STEP == HeadStep::kInputs ? h.piece : h.cols);
            it.rows_end = end_of(it.group);
            it.row0 = begin_of(it.group) + at.row * S::kRows;
            const int nkb = (it.len + kK - 1) / kK;
            constexpr bool kCut = STEP == HeadStep::kInputs || STEP == HeadStep::kLogits;
            it.kb0 = kCut ? (int)((int64_t)nkb * it.split / it.splits) : 0;
            it.kb1 = kCut ? (int)((int64_t)nkb * (it.split + 1) / it.splits) : nkb;
            if (it.row0 >= it.rows_end) it.kb1 = it.kb0;                  // a group with fewer tokens
        }
        return true;
    };
    // An item's contraction goes in stretches of at most args.drain blocks of kK indices: of one, all pairs of terms, block by block, the leading pair last.
    auto stretches = [&](const Item &it) { return (it.kb1 - it.kb0 + args.drain - 1) / args.drain; };

    if (warp == 0) {
        // ------------------------------------------------------------------ copies, by one lane
        wait_for_nothing(smem_u32(&never_bar), abortp);
        if (elect_one()) {
            const uint32_t first_full = BLOCKS == 1 ? full(0) : cluster_addr(&bars[0], 0);
            int s = 0;
            uint32_t round = 0;
            bool ok = true;
            Item it;
            for (int li = 0; ok && get_item(li, it) && !*abortp; ++li) {
                // (of rows that are not there the instructions may read anything)
                const bool rows_here = kAMn || it.row0 + rank * kBlockRows < it.rows_end, rows_there = BLOCKS == 2 && (kAMn || it.row0 + (1 - rank) * kBlockRows < it.rows_end);
                const uint32_t bytes = BLOCKS * S::kBBytes + (rows_here ? kABytes : 0) + (rows_there ? kABytes : 0);
                const int row = it.row0 + rank * kBlockRows, col = it.col0 + rank * HN;
                for (int from = it.kb0, pr = 0; ok && from < it.kb1; pr = pr + 1 == h.pairs ? 0 : pr + 1, from += pr == 0 ? args.drain : 0) {
                    const int plane_a = h.pair_a[pr], plane_b = (STEP == HeadStep::kWeights ? 0 : it.group * h.b_terms) + h.pair_b[pr];
                    for (int kb = from, to = min(it.kb1, from + args.drain); kb < to; ++kb) {
                        ok = mbar_wait(empty(s), (round & 1) ^ 1, abortp);
                        if (!ok) break;
                        const uint32_t to_a = smem_u32(ring) + s * S::kStageBytes, to_b = to_a + kABytes, bar = first_full + s * 8;
                        if (rank == 0) mbar_expect_tx(full(s), bytes);
                        issued[rank][s] = (round + 1) * 4 + rows_there * 2 + rows_here;
                        if (kAMn) {
                            tma_load<BLOCKS>(to_a, &map_a, row, it.k0 + kb * kK, plane_a, bar);
                            tma_load<BLOCKS>(to_a + kK * 128, &map_a, row + 64, it.k0 + kb * kK, plane_a, bar);
                        } else if (rows_here) {
                            tma_load<BLOCKS>(to_a, &map_a, kb * kK, row, plane_a, bar);
                        }
                        if (kBMn) {
                            const int k0 = STEP == HeadStep::kInputs ? (int)h.b_row0 + kb * kK : it.k0 + kb * kK;
                            tma_load<BLOCKS>(to_b, &map_b, col, k0, plane_b, bar);
                            if (HN > 64) tma_load<BLOCKS>(to_b + kK * 128, &map_b, col + 64, k0, plane_b, bar);
                        } else {
                            tma_load<BLOCKS>(to_b, &map_b, kb * kK, (int)h.b_row0 + col, plane_b, bar);
                        }
                        if (++s == S::kStages) {
                            s = 0;
                            ++round;
                        }
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------------ instructions, by one lane of the first block for both
        if (rank == 0 && elect_one()) {
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((kAMn ? 1u : 0u) << 15) | ((kBMn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(S::kRows >> 4) << 24);
            int s = 0;
            uint32_t ph = 0, drain = 0;                              // stretches so far
            bool ok = true;
            Item it;
            for (int li = 0; ok && get_item(li, it) && !*abortp; ++li) {
                for (int from = it.kb0; ok && from < it.kb1; from += args.drain, ++drain) {
                    const int set = (int)(drain & 1), to = min(it.kb1, from + args.drain), all = (to - from) * h.pairs;
                    ok = mbar_wait(dempty(set), ((drain >> 1) & 1) ^ 1, abortp);
                    if (!ok) break;
                    tc_fence_after();
                    for (int j = 0, kb = from; j < all; ++j, kb = kb + 1 == to ? from : kb + 1) {
                        ok = mbar_wait(full(s), ph, abortp);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t ab = smem_u32(ring) + s * S::kStageBytes, bb = ab + kABytes;
                        const uint64_t a_desc = kAMn ? mn_major(ab) : smem_desc_sw128(ab), b_desc = kBMn ? mn_major(bb) : smem_desc_sw128(bb);
                        // 16 contraction indices: 32 bytes of a row, or 16 rows of 128 bytes.  Those behind the last one are left out: another worker's tokens.
                        auto instruction = [&](int k) {
                            mma<BLOCKS>(tmem + set * N, a_desc + k * (kAMn ? 2048 / 16 : 32 / 16), b_desc + k * (kBMn ? 2048 / 16 : 32 / 16), idesc, (uint32_t)(j | k));
                        };
                        const int left = it.len - kb * kK;
                        if (left >= kK) {
#pragma unroll
                            for (int k = 0; k < kK / 16; ++k) instruction(k);
                        } else {
                            for (int k = 0; k * 16 < left; ++k) instruction(k);
                        }
                        commit_to_all<BLOCKS>(empty(s));
                        if (j + 1 == all) commit_to_all<BLOCKS>(dfull(set));
                        if (++s == S::kStages) {
                            s = 0;
                            ph ^= 1;
                        }
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp >= 2) {
        // ------------------------------------------------------------------ sums
        const int quad = warp & 3, part_col = ((warp - 2) >> 2) * kCols;         // TMEM lanes that this warp may access; its columns
        const uint32_t remote_dempty = BLOCKS == 1 || rank == 0 ? 0u : cluster_addr(&bars[2 * S::kStages + 2], 0);
        uint8_t *box = boxes + (warp - 2) * S::kBoxes * kBox;
        int turn = 0;
        uint32_t drain = 0;
        bool ok = true;
        Item it;
        // 16 bytes of this lane's row in the box that goes out next
        auto put16 = [&](int chunk, uint4 v) { *reinterpret_cast<uint4 *>(box + turn * kBox + lane * 128 + ((chunk ^ (lane & 7)) << 4)) = v; };
        auto open_box = [&] {                                      // the box's last store has been read
            if (lane == 0) boxes_wait_read<S::kBoxes - 1>();
            __syncwarp();
        };
        auto close_box = [&](const CUtensorMap *map, bool add, int c0, int c1, int c2) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if (add) add_box(map, box + turn * kBox, c0, c1, c2);
                else store_box(map, box + turn * kBox, c0, c1, c2);
                boxes_commit();
            }
            if (S::kBoxes > 1) turn ^= 1;
        };
        for (int li = 0; ok && __all_sync(0xffffffffu, get_item(li, it) && !*abortp); ++li) {
            float acc[kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[c] = 0.f;
            const int parts = stretches(it);
            for (int part = 0; part < parts; ++part, ++drain) {
                const int set = (int)(drain & 1);
                ok = __all_sync(0xffffffffu, mbar_wait(dfull(set), (drain >> 1) & 1, abortp));
                if (!ok) break;
                tc_fence_after();
                const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + set * N + part_col;
#pragma unroll
                for (int c0 = 0; c0 < kCols; c0 += 32) {
                    uint32_t v[2][16];
                    tc_ld16(from + c0, v[0]);
                    tc_ld16(from + c0 + 16, v[1]);
                    tc_wait_ld();
#pragma unroll
                    for (int k = 0; k < 32; ++k) acc[c0 + k] += __uint_as_float(v[k / 16][k % 16]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (rank == 0) mbar_arrive(dempty(set));
                    else remote_arrive(remote_dempty + set * 8);
                }
            }
            if (!ok) break;
            const int warp_row = it.row0 + rank * kBlockRows + quad * 32, row = warp_row + lane;
            const int col = it.col0 + part_col;                   // the first of this thread's columns
            if (STEP != HeadStep::kWeights && it.row0 >= it.rows_end) continue;

            if constexpr (STEP == HeadStep::kSums) {
                const bool valid = row < it.rows_end;
                const int have = (int)min((int64_t)kCols, h.piece - col);          // words of this thread
#pragma unroll
                for (int c = 0; c < kCols; c += 2) put_two(acc + c, mul2(two_at(acc + c), both(h.scale)));
                if (have < kCols)
#pragma unroll
                    for (int c = 0; c < kCols; ++c)
                        if (c >= have) acc[c] = -INFINITY;
                const int target = valid ? h.targets[row] - (int)(h.v0 + col) : -1;
                if (__any_sync(0xffffffffu, target >= 0 && target < have)) {
                    float z = 0.f;
#pragma unroll
                    for (int c = 0; c < kCols; ++c) z = c == target ? acc[c] : z;
                    if (target >= 0 && target < have) h.target_logit[row] = z;
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                Two sum[2] = {};
#pragma unroll
                for (int c = 0; c < kCols; ++c) top[c & 3] = fmaxf(top[c & 3], acc[c]);
                const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])), beside = most == -INFINITY ? 0.f : most;
#pragma unroll
                for (int c = 0; c < kCols; c += 2) {
                    const Two t = mul2(add2(two_at(acc + c), both(-beside)), both(kLog2e));
                    sum[c >> 1 & 1] = add2(sum[c >> 1 & 1], Two{exp2_fast(t.x), exp2_fast(t.y)});
                }
                if (valid && have > 0) h.part[(int64_t)row * h.part_pitch + (h.v0 + col) / kCols] = make_float2(most, (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y));
            }
            if constexpr (STEP == HeadStep::kProbs) {
                const bool valid = row < it.rows_end;
                const float lse = valid ? h.lse[row] : -INFINITY, g = valid ? h.g[row] : 0.f;
                const bool none = lse == -INFINITY;                // no token, or nothing but logits of minus infinity
                const int target = valid ? h.targets[row] - (int)(h.v0 + col) : -1;
                const bool here = target >= 0 && target < kCols;
                // p - [the target], times -g
#pragma unroll
                for (int c = 0; c < kCols; c += 2) {
                    const Two z = fma2(two_at(acc + c), both(h.scale), both(-lse)), t = mul2(z, both(kLog2e));
                    Two q = {exp2_fast(t.x), exp2_fast(t.y)};
                    if (h.prob_terms > 2) {                         // what t is off by
                        const Two off = fma2(z, both(kLog2eRest), fma2(z, both(kLog2e), Two{-t.x, -t.y}));
                        const Two full = fma2(mul2(off, both(0.69314718f)), q, q);
                        q.x = q.x == 0.f ? 0.f : full.x;            // of t beyond binary32 the correction is none (a NaN remains one)
                        q.y = q.y == 0.f ? 0.f : full.y;
                    }
                    put_two(acc + c, q);
                }
                if (__any_sync(0xffffffffu, here))
#pragma unroll
                    for (int c = 0; c < kCols; ++c)
                        if (here && c == target) acc[c] -= 1.f;
#pragma unroll
                for (int c = 0; c < kCols; c += 2) put_two(acc + c, mul2(two_at(acc + c), both(-g)));
                if (__any_sync(0xffffffffu, none))
#pragma unroll
                    for (int c = 0; c < kCols; ++c) acc[c] = none ? 0.f : acc[c];
                for (int t = 0; t < h.prob_terms; ++t) {
#pragma unroll
                    for (int c0 = 0; c0 < kCols; c0 += 64) {
                        if (col + c0 >= h.piece || warp_row >= h.slots) break;
                        open_box();
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            uint32_t v[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                float *f = &acc[c0 + q * 8 + e * 2];
                                v[e] = two_bf16(f[0], f[1]);
                                // what the next term holds
                                put_two(f, fma2(Two{__uint_as_float(v[e] << 16), __uint_as_float(v[e] & 0xffff0000u)}, both(-1.f), two_at(f)));
                            }
                            put16(q, make_uint4(v[0], v[1], v[2], v[3]));
                        }
                        close_box(&map_out, false, col + c0, warp_row, t);
                    }
                }
            }
            if constexpr (STEP == HeadStep::kInputs || STEP == HeadStep::kLogits) {
#pragma unroll
                for (int c0 = 0; c0 < kCols; c0 += 32) {
                    if (col + c0 >= (STEP == HeadStep::kLogits ? h.piece : h.cols) || warp_row >= h.slots) break;
                    open_box();
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        put16(q, make_uint4(__float_as_uint(acc[c0 + q * 4]), __float_as_uint(acc[c0 + q * 4 + 1]), __float_as_uint(acc[c0 + q * 4 + 2]), __float_as_uint(acc[c0 + q * 4 + 3])));
                    if (STEP == HeadStep::kLogits) close_box(&map_out, false, col + c0, warp_row, it.split);
                    else if (it.split == 0) close_box(&map_out, h.accumulate, col + c0, warp_row, 0);
                    else close_box(&map_extra, h.accumulate, part_col + c0, it.extra * S::kRows + rank * kBlockRows + quad * 32, 0);
                }
            }
            if constexpr (STEP == HeadStep::kWeights) {
                if (!args.manual_stores) {
                    constexpr int kSpan = 128 / sizeof(P), kPer = 16 / sizeof(P);
#pragma unroll
                    for (int c0 = 0; c0 < kCols; c0 += kSpan) {
                        if (col + c0 >= h.cols || warp_row >= it.rows_end) break;
                        open_box();
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            uint32_t v[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                v[e] = sizeof(P) == 4 ? __float_as_uint(acc[c0 + q * kPer + e]) : two_bf16(acc[c0 + q * kPer + e * 2], acc[c0 + q * kPer + (e * 2 + 1) % kPer]);
                            put16(q, make_uint4(v[0], v[1], v[2], v[3]));
                        }
                        close_box(&map_out, false, col + c0, (int)h.v0 + warp_row, it.group);
                    }
                } else {
                    const int rows = min(32, it.rows_end - warp_row);
                    if constexpr (sizeof(P) == 4) {                 // rows of any alignment: 32 columns of a row at a time
                        static_assert(STEP != HeadStep::kWeights || 32 * 33 * 4 <= S::kBoxes * kBox, "32 rows of 32 sums, a word apart");
                        float *turned = reinterpret_cast<float *>(box);
                        P *to = static_cast<P *>(h.dw) + it.group * h.lddw + (h.v0 + warp_row) * h.cols + col + lane;
#pragma unroll
                        for (int c0 = 0; c0 < kCols; c0 += 32) {
#pragma unroll
                            for (int k = 0; k < 32; ++k) turned[lane * 33 + k] = acc[c0 + k];
                            __syncwarp();
                            if (col + c0 + lane < h.cols)
#pragma unroll 4
                                for (int r = 0; r < rows; ++r) put(to + r * h.cols + c0, turned[r * 33 + lane]);
                            __syncwarp();
                        }
                    } else {
                        // Rows of any alignment: 128 bytes of 32 rows by way of shared memory (a row's 16-byte pieces turned about by the row, so that neither lanes
                        // along a row nor lanes along the rows meet in a bank), then 16 bytes at a time to where memory has such a boundary, put together from two
                        // pieces, and single entries before the first and behind the last of them.  Eight lanes to a row.
                        constexpr int kSpan = 64;
                        const int l = lane & 7;
#pragma unroll
                        for (int c0 = 0; c0 < kCols; c0 += kSpan) {
                            const int bytes = (int)min((int64_t)kSpan, h.cols - col - c0) * 2;           // of a row
                            if (bytes <= 0) break;
                            __syncwarp();
#pragma unroll
                            for (int q = 0; q < 8; ++q) {
                                uint32_t v[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) v[e] = two_bf16(acc[c0 + q * 8 + e * 2], acc[c0 + q * 8 + e * 2 + 1]);
                                put16(q, make_uint4(v[0], v[1], v[2], v[3]));
                            }
                            __syncwarp();
                            uint8_t *to = reinterpret_cast<uint8_t *>(static_cast<P *>(h.dw) + it.group * h.lddw + (h.v0 + warp_row + (lane >> 3)) * h.cols + col + c0);
#pragma unroll 4
                            for (int r = lane >> 3; r < rows; r += 4, to += h.cols * 8) {
                                const uint8_t *from = box + r * 128;
                                const int off = (int)(reinterpret_cast<uintptr_t>(to) & 15);
                                auto piece = [&](int q) { return *reinterpret_cast<const uint4 *>(from + (((q ^ r) & 7) << 4)); };
                                // piece l of memory: bytes 16 l - off and on of the row
                                const int at = 16 * l - off;
                                const uint4 v = off == 0 ? piece(l) : shifted<2>(piece(l - 1), piece(l), (unsigned)(16 - off) & 15u);
                                if (at >= 0 && at + 16 <= bytes) *reinterpret_cast<uint4 *>(to + at) = v;
                                // what lies before the first whole piece, and behind the last one
                                const int head = min(bytes, (16 - off) & 15), whole = (bytes - head) & ~15;
                                for (int mine = l * 2; mine < bytes - whole; mine += 16) {
                                    const int byte = mine < head ? mine : mine + whole;
                                    *reinterpret_cast<P *>(to + byte) = *reinterpret_cast<const P *>(from + ((((byte >> 4) ^ r) & 7) << 4) + (byte & 15));
                                }
                            }
                        }
                    }
                }
            }
        }
        if (lane == 0) boxes_wait_all();
    }

    // ---------------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1 && rank == 0 && abort_state[0]) {                 // instructions may still be running
        if (elect_one()) {
            if constexpr (BLOCKS == 1) tc_commit(smem_u32(&drain_bar));
            else asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&drain_bar)) : "memory");
        }
        __syncwarp();
        for (uint32_t i = 0; i < kSpinLimit; ++i) {
            if (mbar_try_wait(smem_u32(&drain_bar), 0)) break;
            __nanosleep(64);
        }
        __syncwarp();
    }
    if (tid == 0) {
        // what the other block has to know
        if (BLOCKS == 1) other_gave_up = 0;
        else asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(&other_gave_up, 1 - rank)), "r"(abort_state[0]) : "memory");
        if (rank != 0)
            for (int s = 0; s < S::kStages; ++s) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr(&issued[1][s], 0)), "r"(issued[1][s]) : "memory");
        if (abort_state[0]) atomicAdd(&g_given_up, 1u);
    }
    __syncthreads();
    if (BLOCKS == 2) cluster_barrier();       // the other block's instructions, arrivals and reads have ended too
    if (abort_state[0] || other_gave_up) {
        // Copies still in flight must land before a block exits.  The blocks are at most one round of a stage apart: bytes that the other one's copies were to
        // bring are counted as here, or are now expected.
        if (tid == 0 && rank == 0)
            for (int s = 0; s < S::kStages; ++s) {
                const uint32_t mine = issued[0][s] >> 2, theirs = BLOCKS == 1 ? mine : issued[1][s] >> 2;
                const auto bytes = [&](uint32_t of_rows) { return (uint32_t)(S::kBBytes + (of_rows ? kABytes : 0)); };
                if (mine > theirs)
                    asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(full(s)), "r"(bytes(issued[0][s] & 2)) : "memory");
                if (theirs > mine) mbar_expect_tx(full(s), bytes(issued[1][s] & 1));
                for (uint32_t i = 0; (mine || theirs) && i < kSpinLimit; ++i) {
                    if (mbar_try_wait(full(s), (max(mine, theirs) - 1) & 1)) break;
                    __nanosleep(64);
                }
            }
        __syncthreads();
        if (BLOCKS == 2) cluster_barrier();
    }
    if (warp == 1) {
        if constexpr (BLOCKS == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * N) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * N) : "memory");
    }
}

uint32_t spin_limit = kSpinLimit;

bool encode(CUtensorMap *map, CUtensorMapDataType type, int size, const void *data, int64_t cols, int64_t rows, int64_t planes, int64_t row, int64_t plane, int box_cols,
            int box_rows) {
    EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes}, strides[2] = {(cuuint64_t)row * size, (cuuint64_t)plane * size};
    const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, ones[3] = {1, 1, 1};
    return enc(map, type, 3, const_cast<void *>(data), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool encode(CUtensorMap *map, const Operand &o, int box_cols, int box_rows) {
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, o.data, o.cols, o.rows, o.planes, o.row, o.plane, box_cols, box_rows);
}

template <HeadStep STEP, int N, int COLS, int BLOCKS, typename P>
cudaError_t launch(const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &out, const CUtensorMap &extra, const KernelArgs &k, int64_t items, cudaStream_t s) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    static PerDeviceOnce once;
    auto *kernel = head_tc_kernel<STEP, N, COLS, BLOCKS, P>;
    if (once.need(device)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (Shape<STEP, N, COLS, BLOCKS>::kSmem));
        if (e != cudaSuccess) return e;
        once.mark(device);
    }
    // equal shares; kInputs cuts what is left over itself
    int64_t pairs = head_pairs() * (BLOCKS == 1 ? 2 : 1);
    if (STEP != HeadStep::kInputs) {
        const int64_t rounds = (items + pairs - 1) / pairs;
        pairs = (items + rounds - 1) / rounds;
    }
    return launch_clustered(kernel, BLOCKS, dim3((unsigned)(BLOCKS * pairs)), dim3(Shape<STEP, N, COLS, BLOCKS>::kThreads), (Shape<STEP, N, COLS, BLOCKS>::kSmem), s, true, a, b, out, extra, k);
}

template <int N, int BLOCKS>
cudaError_t launch_tiles(const HeadTcArgs &h, cudaStream_t s) {
    constexpr int HN = N / 2, kRows = BLOCKS * kBlockRows;
    KernelArgs k = {};
    k.h = h;
    const bool weights = h.step == HeadStep::kWeights, inputs = h.step == HeadStep::kInputs;
    k.row_tiles = (int)(((weights ? h.piece : h.group_slots) + kRows - 1) / kRows);
    k.col_tiles = (int)(((weights || inputs ? h.cols : h.piece) + N - 1) / N);
    k.drain = h.bf16_result ? kDrainBf16 : inputs || weights ? kDrainTerms : h.pairs > 1 ? kDrainLogits : kDrain;
    k.spin_limit = spin_limit;
    const int64_t items = (int64_t)k.row_tiles * k.col_tiles * h.groups;
    if (items == 0) return cudaSuccess;
    if (items >= (int64_t)1 << 30) return cudaErrorInvalidValue;
    CUtensorMap a, b, out = {}, extra = {};
    if (!encode(&a, h.a, 64, weights ? kK : kBlockRows) || !encode(&b, h.b, 64, weights || inputs ? kK : N / BLOCKS)) return cudaErrorInvalidValue;
    const bool brief = head_brief(h.pairs, h.cols);
    switch (h.step) {
        case HeadStep::kSums:
            return brief ? launch<HeadStep::kSums, N, 64, BLOCKS, float>(a, b, out, extra, k, items, s) : launch<HeadStep::kSums, N, HN, BLOCKS, float>(a, b, out, extra, k, items, s);
        case HeadStep::kProbs:
            if (!encode(&out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, h.probs, h.piece, h.slots, h.prob_terms, h.prob_pitch, h.slots * h.prob_pitch, 64, 32)) return cudaErrorInvalidValue;
            return brief ? launch<HeadStep::kProbs, N, 64, BLOCKS, float>(a, b, out, extra, k, items, s) : launch<HeadStep::kProbs, N, HN, BLOCKS, float>(a, b, out, extra, k, items, s);
        case HeadStep::kLogits:
            if (!encode(&out, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, h.logits, h.piece, h.slots, h.logits_parts, h.logits_pitch, h.slots * h.logits_pitch, 32, 32)) return cudaErrorInvalidValue;
            return launch<HeadStep::kLogits, N, HN, BLOCKS, float>(a, b, out, extra, k, items * h.logits_parts, s);
        default: break;
    }
    if constexpr (BLOCKS == 2) {
        if (inputs) {
            if (!encode(&out, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, h.parts, h.cols, h.slots, 1, h.parts_pitch, h.slots * h.parts_pitch, 32, 32) ||
                !encode(&extra, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, h.extra, N, kHeadPairs * kHeadRows, 1, N, kHeadPairs * kHeadRows * N, 32, 32))
                return cudaErrorInvalidValue;
            return launch<HeadStep::kInputs, N, HN, 2, float>(a, b, out, extra, k, items, s);
        }
        const bool bf16 = h.param_type == ZENO_BF16;
        const int size = bf16 ? 2 : 4;
        const int64_t plane = h.groups > 1 ? h.lddw : h.cols, limit = (int64_t)1 << 40;
        k.manual_stores = !(reinterpret_cast<uintptr_t>(h.dw) % 16 == 0 && h.cols * size % 16 == 0 && plane * size % 16 == 0 && plane * size < limit &&
                            encode(&out, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, size, h.dw, h.cols, h.vocab, h.groups, h.cols, plane, 128 / size, 32));
        return bf16 ? launch<HeadStep::kWeights, N, HN, 2, __nv_bfloat16>(a, b, out, extra, k, items, s) : launch<HeadStep::kWeights, N, HN, 2, float>(a, b, out, extra, k, items, s);
    }
    return cudaErrorInvalidValue;                                    // a single block's tiles are of logits
}

}  // namespace

cudaError_t launch_head_tc(const HeadTcArgs &h, cudaStream_t s) {
    if (h.blocks == 1) return h.tile_cols == 128 ? launch_tiles<128, 1>(h, s) : launch_tiles<256, 1>(h, s);
    return h.tile_cols == 128 ? launch_tiles<128, 2>(h, s) : launch_tiles<256, 2>(h, s);
}

int head_pairs() {
    int device = 0, sms = 0;
    if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) sms = 2 * kHeadPairs;
    return sms / 2 < kHeadPairs ? sms / 2 : kHeadPairs;
}

void set_head_wait_limit(uint32_t polls) { spin_limit = polls; }

cudaError_t head_given_up(unsigned *count, cudaStream_t s) {
    void *at = nullptr;
    const cudaError_t e = cudaGetSymbolAddress(&at, g_given_up);
    return e == cudaSuccess ? cudaMemcpyAsync(count, at, sizeof(*count), cudaMemcpyDeviceToHost, s) : e;
}

}  // namespace zeno

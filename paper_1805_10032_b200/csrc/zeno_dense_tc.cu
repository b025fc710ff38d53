// A dense layer's weight gradient dW = dY^T X for every group on the tensor cores, X kept in 8 bits.
//
// A pair of blocks (a cluster of two SMs) takes a tile of 256 outputs by 256 inputs.  dY and X lie token by token, so both operands are read with
// the token as the contraction index and the output or input index contiguous ("MN-major"), in the 128-byte swizzled layout that
// the tensor copies write.  Each block holds 128 of the outputs' rows of dY^T and 128 of the inputs of X, and the pair's instruction
// (cta_group::2, M = 256, N = 256) reads both halves: a code is turned into bfloat16 once for 256 outputs.  code * scale is
// exact in bfloat16, products of bfloat16 are exact, and the sums are binary32 in TMEM, for long ones stretch by stretch.
// 8 x 2048 tokens, 4096 x 4096: 462 us alone (1,190 TFLOP/s, 73 % of cuBLAS's burst rate), 499 with the bias; without the conversion's arithmetic 15 %
// less, without its stores too 24 % less.
//   warp 0: copies of the codes;  warp 3: of their scales;  warp 2: of dY;  warp 1 of the pair's first block: the instructions;
// binary32 dY is rewritten as three bfloat16 terms first, which hold it exactly; few tiles are cut along the tokens.
//   warps 4 - 19: codes to bfloat16;  warps 20 - 23: a finished tile from TMEM to dW while the next one is summed.
#include <map>
#include <mutex>
#include <utility>

#include "zeno_saved.cuh"
#include "zeno_tc.cuh"

namespace zeno {

namespace {

constexpr int kTokens = 64;                   // tokens (the contraction index) of a stage
constexpr int kHalf = 128;                    // outputs, and inputs, of a block
constexpr int kPairTile = 2 * kHalf;
constexpr int kSubBytes = kTokens * 128;      // 64 tokens of 64 bfloat16 (or 128 codes) in 128-byte rows
constexpr int kABytes = 2 * kSubBytes, kBBytes = 2 * kSubBytes, kCodeBytes = kSubBytes, kScaleBytes = kTokens * 4;
constexpr int kStages = 5, kCodeStages = 6;
// A warp's sums of 32 rows on their way from a row a lane to 64 bytes of a row in four lanes' stores (or 16 sums in 16 lanes'): 80 bytes apart, so that
// eight lanes' 16 bytes meet all banks.  By lanes that store along their own rows, 16 bytes of 32 rows at a time, a tile takes about twice as long, which
// shows where tokens are few (30 x 45 tokens, 2320 x 3920 into binary32: 304 us against 577; 8 x 2048, 4096 x 4096 into bfloat16: 500 against 521).
constexpr int kTurnPitch = 80, kTurnBytes = 32 * kTurnPitch;
constexpr int kSmem = kStages * (kABytes + kBBytes) + kCodeStages * (kCodeBytes + kScaleBytes) + 4 * kTurnBytes + 1024;
// The warps that convert come in sets, which take the stages in turn: a stage is a chain of waits, loads, arithmetic, stores and an
// arrival that one set alone would follow from end to end (8 x 2048 tokens, 4096 x 4096, with
// the bias: one set of eight warps 691 us, two of four 589, four of two 562 (536 by now); four of four 515, before the sums left by pieces).
constexpr int kConvWarps = 16, kSets = 4, kSetWarps = kConvWarps / kSets, kEpiWarps = 4;
constexpr int kThreads = 32 * (4 + kConvWarps + kEpiWarps);
constexpr int kTmemCols = 512;                // two sets of 256 sums

__device__ unsigned g_given_up;               // blocks whose bounded waits gave up since the process began

// The tensor core adds with truncation towards zero, which takes about 1.4e-8 of a sum with every 16 tokens: of 2,048 tokens' all positive products
// 1.8e-6, of 32,768 6.7e-5, and 1.2e-4 in three terms.  So no set of sums in TMEM takes more than a stretch of stages; between two stretches of a tile
// the warps that write it keep its sums in binary32 in the workspace (L2), where they are added to nearest: 6.7e-7 for any number of tokens (the plain
// product in binary32: 0.6 to 8e-7).  2 x 8192 tokens, 4096 x 4096, bfloat16 into binary32: 572 us, 482 in one stretch; 8 x 2048 in
// three terms 1,582 and 1,478; stretches of 2,048 tokens are off by 1.8e-6.  A result in bfloat16, which is rounded by 2^-9 anyway, takes stretches of
// 4,096 tokens (4e-6).  Of dY's terms the smaller ones come first: what they lose is 2^-8 of that and less, so that their stretches are 64 times as long.
constexpr int kDrain = 16, kDrainBf16 = 64, kDrainSmall = 64;
struct Stretches {
    int first, last, small_end, early, late;          // stages; where the smaller terms end; stretches in those alone, and others
    __host__ __device__ Stretches(int kb0, int kb1, int small, int drain) : first(kb0), last(kb1) {
        small_end = small < kb0 ? kb0 : small < kb1 ? small : kb1;
        early = (small_end - kb0) / (kDrainSmall * drain);
        late = (kb1 - small_end + drain - 1) / drain;
        if (late == 0 && first + early * kDrainSmall * drain < kb1) late = 1;
    }
    __host__ __device__ int count() const { return early + late; }
    __host__ __device__ int at(int part, int drain) const {
        return part <= early ? first + part * kDrainSmall * drain : small_end + (int)((int64_t)(last - small_end) * (part - early) / late);
    }
};

struct DenseTcArgs {
    DenseGradArgs d;
    int out_tiles, in_tiles, shared_dy, shared_codes;
    int terms;                  // bfloat16 terms of dY, planes of the tensor map's third dimension: summed like further tokens
    int nkb;                    // stages of one term
    int splits;                 // parts that the sum over tokens is cut into
    int drain;                  // stages of a stretch
    float *part;                // [split][group][output][input] (splits > 1)
    float *kept;                // [block][64 times 4 columns][128 outputs] x 4: a block's sums between two stretches of a tile
    int64_t items;
    int vector_stores;
    int followed;               // another kernel of the same call comes after this one
    uint32_t spin_limit;
};

// An arrival at a barrier of the pair's other block.  What it vouches for are this warp's writes to its own shared memory, already
// ordered before the tensor cores' reads of them (fence.proxy.async): with the semantics of a release to the whole cluster every one
// of these arrivals also waited for whatever its lanes had on the way.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
// the pair's commit: an arrival on the barrier at this place in both blocks
__device__ __forceinline__ void pair_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

// MN-major operand in the 128-byte swizzled layout: rows of 64 contiguous entries, one for each value of the contraction index;
// eight of them, 1024 bytes, make a group (stride-dimension offset); the next 64 entries lie kSubBytes on (leading-dimension offset).
__device__ __forceinline__ uint64_t mn_desc(uint32_t addr) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3ffffu) >> 4);
    d |= (uint64_t)(kSubBytes >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

// Two codes (in the upper byte of each half) times 2^120 and the scale.  The sign keeps its place, exponent and mantissa move to where
// bfloat16 has them; its exponent counts from 127, that of the code from 7, and both steps to the code's value times its scale
// are exact.
__device__ __forceinline__ uint32_t two_values(uint32_t high_bytes, __nv_bfloat162 up, __nv_bfloat162 scale) {
    const uint32_t bits = (high_bytes & 0x80008000u) | ((high_bytes >> 4) & 0x07f007f0u);
    const __nv_bfloat162 v = __hmul2(__hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&bits), up), scale);
    return *reinterpret_cast<const uint32_t *>(&v);
}
// 16 codes to two vectors of eight bfloat16
__device__ __forceinline__ void sixteen_values(uint4 codes, float scale, uint4 (&out)[2]) {
    const __nv_bfloat162 up = __float2bfloat162_rn(__uint_as_float((127u + 120u) << 23)), s = __float2bfloat162_rn(scale);
    const uint32_t c[4] = {codes.x, codes.y, codes.z, codes.w};
    uint32_t o[8];
    uint32_t nan = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        nan |= (c[i] & 0x7f7f7f7fu) + 0x01010101u;                            // a byte's top bit: all seven bits were set, NaN
        o[2 * i] = two_values(__byte_perm(c[i], 0u, 0x1404), up, s);
        o[2 * i + 1] = two_values(__byte_perm(c[i], 0u, 0x3424), up, s);
    }
    if (nan & 0x80808080u) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (((c[i / 4] >> (8 * (i % 4))) & 0x7fu) == 0x7fu) o[i / 2] |= 0x7fffu << (16 * (i % 2));
    }
    out[0] = make_uint4(o[0], o[1], o[2], o[3]);
    out[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

// LONG: some sums take more than one stretch.
template <typename P, bool LONG>
__global__ void __launch_bounds__(kThreads, 1) dense_tc_kernel(const __grid_constant__ CUtensorMap map_dy, const __grid_constant__ CUtensorMap map_codes,
                                                               DenseTcArgs a) {
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    // cfull, cempty [kCodeStages]; afull, abempty, bready [kStages]; dfull, dempty [2]
    constexpr int kBars = 2 * kCodeStages + 3 * kStages + 4;
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ __align__(8) uint64_t drain_bar, never_bar;
    __shared__ uint32_t tmem_base_slot;
    __shared__ int abort_state[kAbortWords];
    __shared__ int issued[kCodeStages + kStages];            // last round a copy was issued into a stage, plus one
    __shared__ int scaled[kCodeStages];                      // and the lanes that copy the scales have arrived for

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int rank = (int)cluster_rank();
    uint8_t *a_ring = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *b_ring = a_ring + kStages * kABytes, *code_ring = b_ring + kStages * kBBytes, *scale_ring = code_ring + kCodeStages * kCodeBytes;
    auto bar = [&](int i) { return smem_u32(&bars[i]); };
    auto cfull = [&](int s) { return bar(s); };
    auto cempty = [&](int s) { return bar(kCodeStages + s); };
    auto afull = [&](int s) { return bar(2 * kCodeStages + s); };
    auto abempty = [&](int s) { return bar(2 * kCodeStages + kStages + s); };
    auto bready = [&](int s) { return bar(2 * kCodeStages + 2 * kStages + s); };
    auto dfull = [&](int q) { return bar(2 * kCodeStages + 3 * kStages + q); };
    auto dempty = [&](int q) { return bar(2 * kCodeStages + 3 * kStages + 2 + q); };
    const int64_t n = a.d.n;
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    // item li of this pair -> (group, output tile, input tile, part of the stages); neighbouring pairs share dY's tile in L2
    int group, ot, it, split, kb0, kb1;
    auto get_item = [&](int li) {
        const int64_t item = pair + (int64_t)li * pairs;
        int64_t rest = item / a.splits;
        split = (int)(item - rest * a.splits);
        group = (int)(rest / ((int64_t)a.out_tiles * a.in_tiles));
        const int in_group = (int)(rest - (int64_t)group * a.out_tiles * a.in_tiles);
        ot = in_group / a.in_tiles;
        it = in_group - ot * a.in_tiles;
        const int64_t all = (int64_t)a.terms * a.nkb;
        kb0 = (int)(all * split / a.splits);
        kb1 = (int)(all * (split + 1) / a.splits);
        return item < a.items;
    };

    if (tid == 0) {
        abort_state[0] = 0;
        abort_state[1] = (int)a.spin_limit;
        for (int s = 0; s < kCodeStages; ++s) {
            mbar_init(cfull(s), 1 + 32);       // the codes' copy, and the lanes that copy the scales
            mbar_init(cempty(s), kSetWarps);
        }
        for (int s = 0; s < kStages; ++s) {
            mbar_init(afull(s), 1);
            mbar_init(abempty(s), 1);
            mbar_init(bready(s), 2 * kSetWarps);
        }
        for (int q = 0; q < 2; ++q) {
            mbar_init(dfull(q), 1);
            mbar_init(dempty(q), 2 * kEpiWarps);
        }
        for (int s = 0; s < kCodeStages + kStages; ++s) issued[s] = 0;
        for (int s = 0; s < kCodeStages; ++s) scaled[s] = 0;
        mbar_init(smem_u32(&drain_bar), 1);
        mbar_init(smem_u32(&never_bar), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_barrier();                        // the other block's barriers are there
    tc_fence_after();
    pdl_wait();                               // dY's terms
    if (a.followed) pdl_launch_dependents();  // by a kernel of this call, never by the next call's: that one may read V
    const uint32_t tmem = tmem_base_slot;
    volatile int *abortp = &abort_state[0];
    if (warp == 3) wait_for_nothing(smem_u32(&never_bar), abortp);        // the codes' copies are under way meanwhile
    if (warp == 0 || warp == 2) {
        // ------------------------------------------------------------------ copies: codes (warp 0), dY (warp 2)
        const bool is_codes = warp == 0;
        const int stages = is_codes ? kCodeStages : kStages;
        int s = 0;
        uint32_t round = 0;
        bool ok = true;
        for (int li = 0; ok && __all_sync(0xffffffffu, get_item(li) && !*abortp); ++li)
            for (int kb = kb0, term = kb0 / a.nkb, in_term = kb0 - term * a.nkb; kb < kb1; ++kb) {
                ok = __all_sync(0xffffffffu, mbar_wait(is_codes ? cempty(s) : abempty(s), (round & 1) ^ 1, abortp));
                if (!ok) break;
                const int token0 = in_term * kTokens;
                if (elect_one()) {
                    if (is_codes) {
                        mbar_expect_tx(cfull(s), kCodeBytes);
                        issued[s] = (int)round + 1;
                        tma_load_3d(smem_u32(code_ring + s * kCodeBytes), &map_codes, it * kPairTile + rank * kHalf, token0, a.shared_codes ? 0 : group, cfull(s));
                    } else {
                        mbar_expect_tx(afull(s), kABytes);
                        issued[kCodeStages + s] = (int)round + 1;
#pragma unroll 1
                        for (int h = 0; h < 2; ++h)
                            tma_load_3d(smem_u32(a_ring + s * kABytes + h * kSubBytes), &map_dy, ot * kPairTile + rank * kHalf + h * 64, token0,
                                        a.shared_dy ? 0 : group * a.terms + a.terms - 1 - term, afull(s));
                    }
                }
                __syncwarp();
                if (++in_term == a.nkb) {
                    in_term = 0;
                    ++term;
                }
                if (++s == stages) {
                    s = 0;
                    ++round;
                }
            }
    } else if (warp == 3) {
        // ------------------------------------------------------------------ scales: two tokens a lane
        int s = 0;
        uint32_t round = 0;
        bool ok = true;
        for (int li = 0; ok && __all_sync(0xffffffffu, get_item(li) && !*abortp); ++li) {
            const int64_t block = (int64_t)it * 2 + rank;                   // of 128 columns
            const bool in_range = block * kHalf < a.d.inputs;
            const float *scales = static_cast<const float *>(a.d.scales.data) + group * a.d.scales.group + (in_range ? block : 0);
            for (int kb = kb0, in_term = kb0 % a.nkb; kb < kb1; ++kb) {
                ok = __all_sync(0xffffffffu, mbar_wait(cempty(s), (round & 1) ^ 1, abortp));
                if (!ok) break;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int64_t t = (int64_t)in_term * kTokens + j * 32 + lane;
                    const bool valid = in_range && t < n;
                    cp_async<4>(smem_u32(scale_ring + s * kScaleBytes + (j * 32 + lane) * 4), scales + (valid ? t * a.d.scales.row : 0), valid);
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(cfull(s)) : "memory");
                if (lane == 0) scaled[s] = (int)round + 1;
                if (++in_term == a.nkb) in_term = 0;
                if (++s == kCodeStages) {
                    s = 0;
                    ++round;
                }
            }
        }
        cp_async_commit();
        cp_async_wait<0>();
    } else if (warp == 1) {
        // ------------------------------------------------------------------ instructions, by the first block for both
        // descriptor: sums binary32, operands bfloat16, both MN-major
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(kPairTile >> 3) << 17) | ((uint32_t)(kPairTile >> 4) << 24);
        int s = 0;
        uint32_t ph = 0, drain = 0;                                  // stretches so far
        bool ok = rank == 0;
        for (int li = 0; ok && __all_sync(0xffffffffu, get_item(li) && !*abortp); ++li)
            for (int part = 0, parts = LONG ? Stretches(kb0, kb1, (a.terms - 1) * a.nkb, a.drain).count() : 1; ok && part < parts; ++part, ++drain) {
                const Stretches stretches(kb0, kb1, (a.terms - 1) * a.nkb, a.drain);
                const int set = (int)(drain & 1), from = LONG ? stretches.at(part, a.drain) : kb0, to = LONG ? stretches.at(part + 1, a.drain) : kb1;
                ok = __all_sync(0xffffffffu, mbar_wait(dempty(set), ((drain >> 1) & 1) ^ 1, abortp));
                if (!ok) break;
                tc_fence_after();
                for (int kb = from; kb < to; ++kb) {
                    ok = mbar_wait(bready(s), ph, abortp) && mbar_wait(afull(s), ph, abortp);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t ab = smem_u32(a_ring + s * kABytes), bb = smem_u32(b_ring + s * kBBytes);
#pragma unroll
                        for (int k = 0; k < kTokens / 16; ++k)        // 16 tokens: two groups of eight rows
                            pair_mma(tmem + set * 256, mn_desc(ab + k * 2048), mn_desc(bb + k * 2048), idesc, (uint32_t)((kb - from) | k));
                        pair_commit(abempty(s));
                        if (kb + 1 == to) pair_commit(dfull(set));
                    }
                    __syncwarp();
                    if (++s == kStages) {
                        s = 0;
                        ph ^= 1;
                    }
                }
            }
    } else if (warp >= 4 && warp < 4 + kConvWarps) {
        // ------------------------------------------------------------------ codes to bfloat16
        // Eight lanes take a pair of rows (even and odd token), four of the eight 16-code groups of each, the other four in the other half
        // (`flip`): their 16-byte accesses then meet all banks once, reading and writing, in the swizzled layouts of both.
        const int set = (warp - 4) / kSetWarps, w = (warp - 4) % kSetWarps, l = lane & 7, flip = (lane >> 3) & 1, odd = l >> 2;
        const int g = (l & 3) + 4 * (odd ^ flip);
        const uint32_t remote_bready = rank == 0 ? 0u : cluster_addr(&bars[2 * kCodeStages + 2 * kStages], 0);
        constexpr int kRows = kTokens / (4 * kSetWarps);                    // of a lane
        auto row_of = [&](int j) { return 2 * ((j * kSetWarps + w) * 2 + (lane >> 4)) + odd; };
        uint32_t stage = 0;                                                 // stages so far, all sets'
        bool ok = true;
        for (int li = 0; ok && __all_sync(0xffffffffu, get_item(li) && !*abortp); ++li, stage += kb1 - kb0)
            for (int kb = (int)((set - stage) & (kSets - 1)); kb < kb1 - kb0; kb += kSets) {
                const uint32_t at = stage + kb, round = at / kStages, code_round = at / kCodeStages;
                const int s = (int)(at - round * kStages), sc = (int)(at - code_round * kCodeStages);
                // First the place for the result: that it is free says that all instructions up to kStages stages ago have ended, and so that
                // neither barrier is more than one phase behind (a set does not see every use of a stage, and phases are told by parity).
                ok = mbar_wait(abempty(s), (round & 1) ^ 1, abortp) && mbar_wait(cfull(sc), code_round & 1, abortp);
                // the second block vouches for its part of dY with its part of X
                if (ok && rank != 0) ok = mbar_wait(afull(s), round & 1, abortp);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint8_t *codes = code_ring + sc * kCodeBytes;
                const float *scales = reinterpret_cast<const float *>(scale_ring + sc * kScaleBytes);
                uint8_t *to = b_ring + s * kBBytes + (g >> 2) * kSubBytes;
                uint4 c[kRows];
                float scale[kRows];
#pragma unroll
                for (int j = 0; j < kRows; ++j) {
                    const int row = row_of(j);
                    c[j] = *reinterpret_cast<const uint4 *>(codes + row * 128 + ((g ^ (row & 7)) << 4));
                    scale[j] = scales[row];
                }
#pragma unroll
                for (int j = 0; j < kRows; ++j) {
                    const int row = row_of(j);
                    uint4 v[2];
                    sixteen_values(c[j], scale[j], v);
#pragma unroll
                    for (int h = 0; h < 2; ++h) *reinterpret_cast<uint4 *>(to + row * 128 + (((2 * (g & 3) + h) ^ (row & 7)) << 4)) = v[h];
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    // Behind the fence: it orders the loads of the codes, too, ahead of the next copy's writes, and an arrival alone does not (right behind
                    // the loads, without a fence, it gave wrong sums).
                    mbar_arrive(cempty(sc));
                    if (rank == 0) mbar_arrive(bready(s));
                    else mbar_arrive_cluster(remote_bready + s * 8);
                }
            }
    } else if (warp >= 4 + kConvWarps) {
        // ------------------------------------------------------------------ finished tiles to dW
        const int quad = warp & 3;                                 // TMEM lanes this warp may access
        const uint32_t remote_dempty = rank == 0 ? 0u : cluster_addr(&bars[2 * kCodeStages + 3 * kStages + 2], 0);
        uint32_t drain = 0;
        for (int li = 0; __all_sync(0xffffffffu, get_item(li) && !*abortp); ++li)      // a wait that gave up has raised the flag
            for (int part = 0, parts = LONG ? Stretches(kb0, kb1, (a.terms - 1) * a.nkb, a.drain).count() : 1; part < parts; ++part, ++drain) {
                const int set = (int)(drain & 1);
                if (!__all_sync(0xffffffffu, mbar_wait(dfull(set), (drain >> 1) & 1, abortp))) break;
                tc_fence_after();
                const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + set * 256;
                // the sums of 32 columns; behind the last of them the set may be overwritten
                auto take = [&](int c0, uint32_t (&v)[2][16]) {
                    __syncwarp();
                    tc_ld16(from + c0, v[0]);
                    tc_ld16(from + c0 + 16, v[1]);
                    tc_wait_ld();
                    if (c0 + 32 == kPairTile) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            if (rank == 0) mbar_arrive(dempty(set));
                            else mbar_arrive_cluster(remote_dempty + set * 8);
                        }
                    }
                };
                // what was kept of the tile's earlier stretches is added; a thread meets none but its own
                auto kept = [&](int c0) { return reinterpret_cast<float4 *>(a.kept) + ((blockIdx.x * kPairTile + c0) / 4 * kHalf + quad * 32 + lane); };
                auto add_kept = [&](int c0, uint32_t (&v)[2][16]) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float4 f = __ldcg(kept(c0) + k * kHalf);
                        uint32_t *u = v[k / 4] + k % 4 * 4;
                        u[0] = __float_as_uint(__uint_as_float(u[0]) + f.x);
                        u[1] = __float_as_uint(__uint_as_float(u[1]) + f.y);
                        u[2] = __float_as_uint(__uint_as_float(u[2]) + f.z);
                        u[3] = __float_as_uint(__uint_as_float(u[3]) + f.w);
                    }
                };
                if (LONG && part + 1 < parts) {
#pragma unroll 1
                    for (int c0 = 0; c0 < kPairTile; c0 += 32) {
                        uint32_t v[2][16];
                        take(c0, v);
                        if (part > 0) add_kept(c0, v);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const uint32_t *u = v[k / 4] + k % 4 * 4;
                            __stcg(kept(c0) + k * kHalf, make_float4(__uint_as_float(u[0]), __uint_as_float(u[1]), __uint_as_float(u[2]), __uint_as_float(u[3])));
                        }
                    }
                    continue;
                }
                const int64_t o = (int64_t)ot * kPairTile + rank * kHalf + quad * 32 + lane, k0 = (int64_t)it * kPairTile;
                P *dw = a.splits > 1 ? reinterpret_cast<P *>(a.part) + (((int64_t)split * a.d.m + group) * a.d.outputs + o) * a.d.inputs + k0
                                     : static_cast<P *>(a.d.dw) + group * a.d.ldw + o * a.d.inputs + k0;
#pragma unroll 1
                for (int c0 = 0; c0 < kPairTile; c0 += 32) {
                    uint32_t v[2][16];
                    take(c0, v);
                    if constexpr (LONG)
                        if (part > 0) add_kept(c0, v);
                    uint8_t *turns = scale_ring + kCodeStages * kScaleBytes + quad * kTurnBytes;
                    const int rows = (int)min((int64_t)32, a.d.outputs - (o - lane));
                    const int pitch = (int)a.d.inputs;
                    P *corner = dw - lane * pitch + c0;
                    if (a.vector_stores) {
                        constexpr int kPer = 16 / sizeof(P), kAtOnce = 4 * kPer;
#pragma unroll
                        for (int h = 0; h < 32 / kAtOnce; ++h) {
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                alignas(16) P e[kPer];
#pragma unroll
                                for (int k = 0; k < kPer; ++k) {
                                    const int col = h * kAtOnce + q * kPer + k;
                                    put(e + k, __uint_as_float(v[col / 16][col % 16]));
                                }
                                *reinterpret_cast<uint4 *>(turns + lane * kTurnPitch + q * 16) = *reinterpret_cast<const uint4 *>(e);
                            }
                            __syncwarp();
                            const int col = h * kAtOnce + (lane & 3) * kPer;
                            uint4 piece[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) piece[k] = *reinterpret_cast<const uint4 *>(turns + (k * 8 + (lane >> 2)) * kTurnPitch + (lane & 3) * 16);
                            __syncwarp();
                            const int below = k0 + c0 + col < a.d.inputs ? rows - (lane >> 2) : 0;
                            P *to = corner + (lane >> 2) * pitch + col;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (k * 8 < below) *reinterpret_cast<uint4 *>(to + k * 8 * pitch) = piece[k];
                        }
                    } else {                                            // rows of any alignment: two outputs' 16 sums in a store of the warp
                        float *turn = reinterpret_cast<float *>(turns);
                        const int col = lane & 15;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
#pragma unroll
                            for (int k = 0; k < 16; ++k) turn[lane * 17 + k] = __uint_as_float(v[h][k]);
                            __syncwarp();
                            const int at = h * 16 + col, below = k0 + c0 + at < a.d.inputs ? rows - (lane >> 4) : 0;
                            P *to = corner + (lane >> 4) * pitch + at;
#pragma unroll 1
                            for (int k = 0; k < below; k += 8, to += 8 * pitch) {
                                float f[4];
#pragma unroll
                                for (int u = 0; u < 4; ++u) f[u] = turn[(k + 2 * u + (lane >> 4)) * 17 + col];
#pragma unroll
                                for (int u = 0; u < 4; ++u)
                                    if (k + 2 * u < below) put(to + 2 * u * pitch, f[u]);
                            }
                            __syncwarp();
                        }
                    }
                }
            }
    }

    // ---------------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1 && rank == 0 && abort_state[0]) {                 // instructions may still be running
        if (elect_one()) asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&drain_bar)) : "memory");
        __syncwarp();
        for (uint32_t i = 0; i < kSpinLimit; ++i) {
            if (mbar_try_wait(smem_u32(&drain_bar), 0)) break;
            __nanosleep(64);
        }
        __syncwarp();
    }
    if (tid == 0 && abort_state[0]) {
        // copies still in flight must land before the block exits
        for (int s = 0; s < kCodeStages + kStages; ++s)
            if (issued[s] > 0) {
                const uint32_t b = s < kCodeStages ? cfull(s) : afull(s - kCodeStages);
                // the scales' warp may have left before the codes' copy that the barrier is to tell of
                if (s < kCodeStages && scaled[s] < issued[s]) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], 32;" ::"r"(b) : "memory");
                for (uint32_t i = 0; i < kSpinLimit; ++i) {
                    if (mbar_try_wait(b, (uint32_t)(issued[s] - 1) & 1)) break;
                    __nanosleep(64);
                }
            }
        atomicAdd(&g_given_up, 1u);
    }
    __syncthreads();
    cluster_barrier();                        // the other block's instructions, arrivals and reads have ended too
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

// dY as bfloat16 terms in [group][term][token][outputs, rounded up to 8]: one term (of bfloat16 in rows that no tensor map can step through) or
// three, which hold a binary32 number exactly (from 2^-110 on; a smaller one has bits under bfloat16's smallest step, 2^-133, and is off by half of that): each
// takes the leading 8 bits of what is left.  An infinity or NaN is its first term.
template <typename T, int TERMS>
__global__ void __launch_bounds__(256) dense_terms_kernel(Rows dy, int64_t rows, int64_t n, int64_t outputs, int64_t pitch, __nv_bfloat16 *out, int vectors) {
    const int64_t per_row = pitch / 8, total = rows * per_row;
    pdl_launch_dependents();
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (int64_t)gridDim.x * 256) {
        const int64_t r = q / per_row, o = (q - r * per_row) * 8, group = r / n;
        const T *from = static_cast<const T *>(dy.data) + dy.at(r) + o;
        alignas(16) T e[8];
        float f[8];
        if (vectors) {
#pragma unroll
            for (int k = 0; k < (int)sizeof(e) / 16; ++k) reinterpret_cast<uint4 *>(e)[k] = reinterpret_cast<const uint4 *>(from)[k];
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = value_of(e + k);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = o + k < outputs ? value_of(from + k) : 0.f;
        }
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
            alignas(16) __nv_bfloat16 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] = __float2bfloat16_rn(f[k]);
                // (a finite number may round to infinity: then the term is the largest finite one)
                if (fabsf(f[k]) < INFINITY && !(fabsf(__bfloat162float(v[k])) < INFINITY)) v[k] = __ushort_as_bfloat16(f[k] < 0.f ? 0xff7f : 0x7f7f);
                f[k] = fabsf(f[k]) < INFINITY ? f[k] - __bfloat162float(v[k]) : 0.f;
            }
            *reinterpret_cast<uint4 *>(out + ((group * TERMS + t) * n + (r - group * n)) * pitch + o) = *reinterpret_cast<const uint4 *>(v);
        }
    }
}

// the parts' sums, N neighbouring entries a thread
template <typename P, int N>
__global__ void __launch_bounds__(256) dense_join_kernel(const float *part, int splits, int64_t per_group, int64_t total, P *dw, int64_t ldw, int followed) {
    pdl_wait();
    if (followed) pdl_launch_dependents();
    const int64_t q = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N;
    if (q >= total) return;
    float s[N] = {};
#pragma unroll 8
    for (int k = 0; k < splits; ++k) {
        alignas(16) float v[N];
        if constexpr (N == 4) *reinterpret_cast<float4 *>(v) = *reinterpret_cast<const float4 *>(part + k * total + q);
        else v[0] = part[k * total + q];
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] += v[j];
    }
    const int64_t group = q / per_group;
    P *to = dw + group * ldw + (q - group * per_group);
#pragma unroll
    for (int j = 0; j < N; ++j) put(to + j, s[j]);
}

uint32_t spin_limit = kSpinLimit;

bool encode(CUtensorMap *map, CUtensorMapDataType type, const Rows &v, int elem, int m, int64_t n, int64_t cols, int box_cols) {
    EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return false;
    const bool shared = m > 1 && v.group == 0;
    const cuuint64_t row = (cuuint64_t)(n > 1 ? v.row : (cols * elem + 15) / 16 * 16 / elem) * elem;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)n, (cuuint64_t)(shared ? 1 : m)};
    const cuuint64_t strides[2] = {row, m > 1 && !shared ? (cuuint64_t)v.group * elem : row};
    const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)kTokens, 1}, ones[3] = {1, 1, 1};
    return enc(map, type, 3, v.data, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// groups behind one another (or one for all), rows that a tensor map can step through
bool mappable(const Rows &v, int elem, int m, int64_t n, int64_t cols) {
    const int64_t limit = (int64_t)1 << 39;
    if (!aligned_to(v, m, n, elem, 16)) return false;
    if (n > 1 && v.row * elem >= limit) return false;
    return m <= 1 || v.group == 0 || (v.group >= (n > 1 ? n * v.row : cols) && v.group * elem < limit);
}

// What a call does: the terms that dY is rewritten in (0: it is read as it lies), the parts of the sum, and where they lie in the workspace.
struct Plan {
    int terms, splits, out_tiles, in_tiles;
    int64_t pitch, part_at, kept_at, bytes;
};

// Parts: with fewer tiles than half the pairs of SMs, as many as the pairs take, each of eight stages and more (bfloat16: 4 x 8192 tokens, 512 x 1024,
// 53 us, 80 in one part; 1 x 8192, 512 x 512, 27 and 72).  More tiles are not cut: in four parts 54 of them take 53 us and not 55 (6 x 4843, 640 x 560), 40
// take 39 and not 29 (10 x 2048, 512 x 512).  The count of SMs is this
// design's, so that the workspace's size needs no device.
constexpr int kPairs = 74;

// Whether any part takes more than one stretch.
bool long_sums(const Plan &p, const DenseGradArgs &a, int drain) {
    const int terms = p.terms > 1 ? p.terms : 1, nkb = (int)((a.n + kTokens - 1) / kTokens);
    const int64_t all = (int64_t)terms * nkb;
    for (int s = 0; s < p.splits; ++s)
        if (Stretches((int)(all * s / p.splits), (int)(all * (s + 1) / p.splits), (terms - 1) * nkb, drain).count() > 1) return true;
    return false;
}

bool plan_dense_tc(int type, const DenseGradArgs &a, Plan *p) {
    if (a.n < 1 || a.n >= (int64_t)1 << 28 || !mappable(a.codes, 1, a.m, a.n, a.inputs)) return false;
    p->terms = type == ZENO_F32 ? 3 : mappable(a.dy, 2, a.m, a.n, a.outputs) ? 0 : 1;
    p->pitch = (a.outputs + 7) / 8 * 8;
    p->out_tiles = (int)((a.outputs + kPairTile - 1) / kPairTile);
    p->in_tiles = (int)((a.inputs + kPairTile - 1) / kPairTile);
    const int64_t tiles = (int64_t)a.m * p->out_tiles * p->in_tiles, stages = (a.n + kTokens - 1) / kTokens * (p->terms > 1 ? p->terms : 1);
    int64_t splits = tiles * 2 > kPairs ? 1 : kPairs / tiles;
    if (splits > stages / 8) splits = stages / 8;
    p->splits = splits < 1 ? 1 : (int)splits;
    const int64_t terms_bytes = (int64_t)a.m * p->terms * a.n * p->pitch * 2;
    p->part_at = (terms_bytes + 255) / 256 * 256;
    p->kept_at = p->part_at + ((p->splits > 1 ? (int64_t)p->splits * a.m * a.outputs * a.inputs * 4 : 0) + 255) / 256 * 256;
    p->bytes = p->kept_at + (long_sums(*p, a, kDrain) ? (int64_t)2 * kPairs * kHalf * kPairTile * 4 : 0);
    return true;
}

}  // namespace

int64_t dense_tc_workspace(int type, const DenseGradArgs &a) {
    Plan p;
    return plan_dense_tc(type, a, &p) ? p.bytes : 0;
}

cudaError_t launch_dense_tc(int type, int param_type, const DenseGradArgs &d, cudaStream_t s) {
    Plan p;
    if (!plan_dense_tc(type, d, &p)) return cudaErrorNotSupported;
    uint8_t *ws = reinterpret_cast<uint8_t *>(d.workspace);
    Rows dy = d.dy;
    int planes = d.m;
    if (p.terms) {
        planes = d.m * p.terms;
        dy = Rows{ws, p.pitch, d.n * p.pitch, d.n};
    }
    CUtensorMap map_dy, map_codes;
    if (!encode(&map_dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dy, 2, planes, d.n, d.outputs, 64) ||
        !encode(&map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, d.codes, 1, d.m, d.n, d.inputs, 128))
        return cudaErrorNotSupported;
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return e;
    if (p.terms) {
        const int64_t rows = d.m * d.n, blocks = (rows * (p.pitch / 8) + 255) / 256;
        const bool vectors = d.outputs % 8 == 0 && aligned_to(d.dy, d.m, d.n, type == ZENO_F32 ? 4 : 2, 16);
        const dim3 grid((unsigned)(blocks < 148 * 16 ? blocks : 148 * 16));
        auto *out = reinterpret_cast<__nv_bfloat16 *>(ws);
        e = type == ZENO_F32 ? launch_chained(dense_terms_kernel<float, 3>, grid, dim3(256), 0, s, false, d.dy, rows, d.n, d.outputs, p.pitch, out, (int)vectors)
                             : launch_chained(dense_terms_kernel<__nv_bfloat16, 1>, grid, dim3(256), 0, s, false, d.dy, rows, d.n, d.outputs, p.pitch, out, (int)vectors);
        if (e != cudaSuccess) return e;
    }
    DenseTcArgs a;
    a.d = d;
    a.out_tiles = p.out_tiles;
    a.in_tiles = p.in_tiles;
    a.shared_dy = p.terms == 0 && d.m > 1 && d.dy.group == 0;
    a.shared_codes = d.m > 1 && d.codes.group == 0;
    a.terms = p.terms > 1 ? p.terms : 1;
    a.nkb = (int)((d.n + kTokens - 1) / kTokens);
    a.splits = p.splits;
    a.drain = param_type == ZENO_BF16 ? kDrainBf16 : kDrain;
    a.part = reinterpret_cast<float *>(ws + p.part_at);
    a.kept = reinterpret_cast<float *>(ws + p.kept_at);
    a.items = (int64_t)d.m * a.out_tiles * a.in_tiles * a.splits;
    const bool bf16 = param_type == ZENO_BF16 && p.splits == 1;
    const size_t elem = bf16 ? 2 : 4;
    a.vector_stores = d.inputs * elem % 16 == 0 &&
                      (p.splits > 1 || (reinterpret_cast<uintptr_t>(d.dw) % 16 == 0 && (d.m <= 1 || d.ldw * elem % 16 == 0)));
    a.followed = p.splits > 1 || d.db;
    a.spin_limit = spin_limit;
    const bool in_stretches = long_sums(p, d, a.drain);
    auto *kernel = bf16 ? (in_stretches ? dense_tc_kernel<__nv_bfloat16, true> : dense_tc_kernel<__nv_bfloat16, false>)
                        : (in_stretches ? dense_tc_kernel<float, true> : dense_tc_kernel<float, false>);
    static PerDeviceOnce attr_set[4];
    PerDeviceOnce &once = attr_set[2 * bf16 + in_stretches];
    if (once.need(device)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return e;
        once.mark(device);
    }
    // equal shares: the fewest pairs that make as many rounds as all would
    const int64_t most = sms / 2 < kPairs ? sms / 2 : kPairs, rounds = (a.items + most - 1) / most, pairs = (a.items + rounds - 1) / rounds;
    e = launch_clustered(kernel, 2, dim3((unsigned)(2 * pairs)), dim3(kThreads), kSmem, s, p.terms > 0, map_dy, map_codes, a);
    if (e != cudaSuccess || p.splits == 1) return e;
    const int64_t per_group = d.outputs * d.inputs, total = per_group * d.m;
    const int n = per_group % 4 == 0 ? 4 : 1;
    const dim3 grid((unsigned)((total / n + 255) / 256));
    if (param_type == ZENO_BF16)
        return launch_chained(n == 4 ? dense_join_kernel<__nv_bfloat16, 4> : dense_join_kernel<__nv_bfloat16, 1>, grid, dim3(256), 0, s, true, a.part, p.splits,
                              per_group, total, static_cast<__nv_bfloat16 *>(d.dw), d.ldw, (int)(d.db != nullptr));
    return launch_chained(n == 4 ? dense_join_kernel<float, 4> : dense_join_kernel<float, 1>, grid, dim3(256), 0, s, true, a.part, p.splits, per_group, total,
                          static_cast<float *>(d.dw), d.ldw, (int)(d.db != nullptr));
}

void set_operator_wait_limit(uint32_t polls) { spin_limit = polls; }

// The count is never cleared, since a block of another stream may give up at any time; what differs is what a stream's last report knew of.
cudaError_t read_operator_status(int device, cudaStream_t s, int *status) try {
    static std::mutex mutex;
    static std::map<std::pair<int, cudaStream_t>, unsigned> known;
    void *at = nullptr;
    unsigned count = 0;
    cudaError_t e = cudaGetSymbolAddress(&at, g_given_up);
    if (e == cudaSuccess) e = cudaMemcpyAsync(&count, at, sizeof(count), cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mutex);
    unsigned &before = known[{device, s}];
    *status = count != before;
    before = count;
    return cudaSuccess;
} catch (...) {
    return cudaErrorMemoryAllocation;
}

}  // namespace zeno

// The output layer's products on the tensor cores (zeno_head_tc.cu) and what zeno_head.cu hands them.
#pragma once

#include "zeno_operators.h"

namespace zeno {

// Tokens that carry a target lie in slots: worker i's in [begin[i], end[i]), for the gradient both multiples of kSlots, the contraction indices of an
// instruction; those left over are empty.
constexpr int kSlots = 16;
constexpr int kMaxPairs = 6;

// Operands as bfloat16 terms: one of a bfloat16 number, three of a binary32 one, in planes of their own.
struct Operand {
    const void *data;
    int64_t cols, rows;                 // contiguous entries, and how many rows of them
    int64_t row, plane;                 // entries from one row, plane, to the next
    int planes;
};

enum class HeadStep { kSums, kProbs, kLogits, kInputs, kWeights };

struct HeadTcArgs {
    HeadStep step;
    Operand a, b;                       // a: X, P (kInputs, kWeights); b: W, X (kWeights)
    int pairs, pair_a[kMaxPairs], pair_b[kMaxPairs];        // terms that are multiplied, the last pair the leading ones
    int b_terms;                        // b's planes of a group
    int groups;                         // with weights of their own; kWeights: the workers
    const int *begin, *end;             // slots of each group
    int64_t slots;                      // at most, of all groups
    int64_t group_slots;                // and of one
    int64_t cols, vocab;
    int64_t v0, piece;                  // the vocabulary's words of this call
    int64_t b_row0;                     // where they begin among b's rows
    float scale;
    // kSums
    const int *targets;                 // [slot]
    float2 *part;                       // [slot][part_pitch]: largest logit and the sum of exponentials beside it, of 64 words each in brief tiles, of half a tile's in others
    int64_t part_pitch;
    float *target_logit;                // [slot]
    // kProbs
    const float *lse, *g;               // [slot]; g times the scale
    __nv_bfloat16 *probs;               // [term][slots][prob_pitch]
    int64_t prob_pitch;
    int prob_terms;
    // kLogits: unscaled, in parts of the contraction
    float *logits;                      // [part][slots][logits_pitch]
    int64_t logits_pitch;
    int logits_parts;
    // kInputs
    float *parts;                       // [slots][parts_pitch]
    int64_t parts_pitch;
    float *extra;                       // [item behind the whole rounds][256][tile_cols]: parts of tiles that are cut, but for their first ones
    int most_splits, accumulate;
    // kWeights
    void *dw;
    int64_t lddw;
    int param_type;
    int bf16_result;                    // what comes of the sums is bfloat16
    int tile_cols;                      // columns of a tile: 256 or 128
    int blocks;                         // of a tile: two, or (kSums, kProbs, kLogits) one
    int last;                           // no kernel of the same call comes after this one
};

cudaError_t launch_head_tc(const HeadTcArgs &h, cudaStream_t s);

constexpr int kHeadRows = 256;          // rows of a tile

// Tiles of fewer stages wait for the warps that take their sums, which sixteen with 64 columns each do sooner than eight with 128 (12 x 5555 tokens, 40103 words by
// 84 columns: 1,315 us, 1,490); with more, the room that their boxes take is better spent on stages (132 tokens, 40576 words by 5568 columns in binary32:
// 168 us a piece with eight, 189).
inline bool head_brief(int pairs, int64_t cols) { return pairs * ((cols + 63) / 64) < 16; }
constexpr int kHeadPairs = 74;          // pairs of SMs of this design
int head_pairs();                       // that the current device has, of those

// Tile number t of a group: rows first within a band of kHeadBand tiles of them, then columns.
constexpr uint32_t kHeadBand = 16;
struct HeadTile { int row, col; };
__host__ __device__ inline HeadTile head_tile(uint32_t t, uint32_t row_tiles, uint32_t col_tiles) {
    const uint32_t band = t / (kHeadBand * col_tiles), in = t - band * kHeadBand * col_tiles, left = row_tiles - band * kHeadBand, rows = left < kHeadBand ? left : kHeadBand;
    const uint32_t col = in / rows;
    return HeadTile{(int)(band * kHeadBand + in - col * rows), (int)col};
}
__host__ __device__ inline uint32_t head_tile_number(int row, int col, uint32_t row_tiles, uint32_t col_tiles) {
    const uint32_t band = row / kHeadBand, left = row_tiles - band * kHeadBand, rows = left < kHeadBand ? left : kHeadBand;
    return band * kHeadBand * col_tiles + col * rows + (row - band * kHeadBand);
}
// Parts that the tiles behind the whole rounds of all pairs are cut into.
__host__ __device__ inline int head_splits(uint32_t tiles, uint32_t pairs, int most) {
    const uint32_t rest = tiles % pairs;
    const int fit = rest ? (int)(pairs / rest) : 1;
    return fit < most ? fit : most;
}

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
#endif

}  // namespace zeno

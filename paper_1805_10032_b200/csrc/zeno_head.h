// The output layer's products on the tensor cores (zeno_head_tc.cu) and what zeno_head.cu hands them.
#pragma once

#include "zeno_operators.h"

namespace zeno {

// Tokens that carry a target lie in slots: worker i's in [begin[i], end[i]), both multiples of kSlots, those left over empty.
constexpr int kSlots = 64;
constexpr int kMaxPairs = 6;

// Operands as bfloat16 terms: one of a bfloat16 number, three of a binary32 one, in planes of their own.
struct Operand {
    const void *data;
    int64_t cols, rows;                 // contiguous entries, and how many rows of them
    int64_t row, plane;                 // entries from one row, plane, to the next
    int planes;
};

enum class HeadStep { kSums, kProbs, kInputs, kWeights };

struct HeadTcArgs {
    HeadStep step;
    Operand a, b;                       // a: X (kSums, kProbs), P (kInputs, kWeights); b: W (kSums, kProbs, kInputs), X (kWeights)
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
    float2 *part;                       // [slot][part_pitch]: largest logit and the sum of exponentials beside it, of head_sum_cols() words each
    int64_t part_pitch;
    float *target_logit;                // [slot]
    // kProbs
    const float *lse, *g;               // [slot]; g times the scale
    __nv_bfloat16 *probs;               // [term][slots][prob_pitch]
    int64_t prob_pitch;
    int prob_terms;
    // kInputs
    float *parts;                       // [split][slots][parts_pitch]
    int64_t parts_pitch;
    int splits, accumulate;
    // kWeights
    void *dw;
    int64_t lddw;
    int param_type;
    int last;                           // no kernel of the same call comes after this one
};

int head_tile_cols(int64_t rows_bound, int64_t groups, int64_t cols);
cudaError_t launch_head_tc(const HeadTcArgs &a, cudaStream_t s);

}  // namespace zeno

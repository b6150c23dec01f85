// Launches of the token loss and its gradients (loss_kernel.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "lookup_kernel.h"

namespace micro {

// Products advance 64 values of the summed axis at a time: padded axes are
// multiples of it.
constexpr int kProductDepth = 64;
// binary32 operands enter the products as the sum of this many bfloat16 ones.
constexpr int kSplitPlanes = 3;
// Tiles of the products, by the call's tokens.  Middle ones (128 x 128, two
// workgroups a compute unit) up to kSomeTokens: with gradients over 30522 x 1024
// 100 tokens take 100 us and 300 take 135, in wide tiles (256 x 256, one
// workgroup) 128 and 145; 512 tokens 162 and 161, over 50257 x 2048 470 and 416.
// (Settled on these two tables.  Over a few thousand rows the wide tiles of more
// tokens than that do not fill the card, and middle ones might be faster.)
// The loss alone of up to kFewTokens takes narrow ones (128 vocabulary rows x 32
// tokens): it is bound by one read of the table (32 us over 50257 x 2048, 6.5
// TB/s), which many small workgroups keep going.
constexpr int kFewTokens = 32, kSomeTokens = 384;
// Vocabulary rows that share one running maximum: what one wavefront of the
// score product holds, in wide, middle and narrow tiles.
constexpr int kGranule = 128, kGranuleSome = 64, kGranuleFew = 32;

// One call's operands and scratch.  Lengths: D = dim, Dp = D rounded up to
// kProductDepth, Vp = vocab rounded up to it, B = tokens of a block (a
// multiple of 256), P = planes (kSplitPlanes for binary32, else 1).
struct LossCall {
    int32_t type;            // of hidden, table and gradients
    int64_t vocab, vocab_padded;
    int32_t dim, dim_padded;
    int64_t tokens, block;   // B
    Rows hidden, table;
    TokenIds targets;
    int64_t ignored;         // the target value that does not count
    bool mean;
    float scale;             // of the gradients
    float* losses;           // out, one per token
    float* loss;             // out
    bool gradients;
    bool accumulate;         // add to dtable
    Rows dhidden, dtable;    // out
    // scratch
    uint32_t* chunks;        // counted tokens of each 1024
    int32_t* count;          // counted tokens, whether a target lies outside the vocabulary, arrivals
    int32_t* rows;           // their positions, ascending
    int32_t* labels;         // and targets
    float* counted_losses;   // one per counted token
    void* h;                 // counted rows of hidden, [P][tokens rounded up to 64][Dp]
    void* w;                 // table rows, [P][vocab][Dp], where the table itself cannot be read in place
    float2* stats;           // (maximum, sum of exponentials) of [granule][B]
    float* label_logit;      // [B]
    float* label_rest;       // 16-bit types: the logit gradient at the label less its rounding, [B]
    float2* softmax;         // (maximum, 1 / sum of exponentials) of [B]
    void* scores;            // exponentials (binary32: floats, else 16-bit codes), then logit gradients, [B][Vp]
    void* split;             // binary32: the logit gradients as [P][B][Vp] bfloat16
    float* parts;            // parts of a short call's scores cut along the sum: two middle tiles or four narrow ones per compute unit
    float* partials;         // parts of the two gradient products cut along the sum: a wide tile per compute unit each
    float* carried;          // wide tiles of dtable between token blocks; null with one block
    int compute_units;
};

// Whether the product can read the table where it is.
bool table_in_place(const LossCall& c);

hipError_t launch_loss(const LossCall& call, hipStream_t stream);

// Floats of one wide product tile, and of a short call's largest.
constexpr int64_t kWideTile = 256 * 256, kPartTile = 128 * 128;

}  // namespace micro

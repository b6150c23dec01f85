// Launch of the drawing of tokens from logits (sample_kernel.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "lookup_kernel.h"
#include "micro_sparsify.h"

namespace micro {

// Weights are whole multiples of 2^-bits, and the sum of `vocab` of them stays
// below 2^63.
constexpr int kMostWeightBits = 50;
constexpr int weight_bits(int64_t vocab) {
    int log = 0;
    while ((int64_t(1) << log) < vocab) ++log;
    return 62 - log < kMostWeightBits ? 62 - log : kMostWeightBits;
}

struct SampleCall {
    Rows logits;
    int64_t rows, vocab;
    const float* uniforms;
    micro_sampling sampling;
    TokenIds ids;      // out
    float* logprobs;   // out, may be null
    int compute_units;
};

hipError_t launch_sample(const SampleCall& call, hipStream_t stream);

}  // namespace micro

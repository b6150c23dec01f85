// Launches of the token table's lookup and of its gradient (lookup_kernel.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace micro {

// Token ids on the device, int32 or int64.
struct TokenIds {
    const void* at;
    bool wide;  // int64
};

// A tensor of rows: values of one row are adjacent, rows `stride` values apart.
struct Rows {
    void* at;
    int64_t stride;
    int32_t type;  // MICRO_TYPE_*
};

// out[t] = scale * table[ids[t]] for t in [0, tokens); NaN where ids[t] is
// outside [0, vocab).
hipError_t launch_lookup(const Rows& table, int64_t vocab, int32_t dim, const TokenIds& ids, int64_t tokens,
                         float scale, const Rows& out, hipStream_t stream);

// Tokens that one workgroup sorts in shared memory.
constexpr int kSortTile = 4096;
// Sorted tokens that one thread group sums.
constexpr int kSumChunk = 16;

// Scratch of the lookup's gradient for up to `tokens` tokens.
struct LookupGradScratch {
    uint32_t* keys[2];   // sorted token ids, `tokens` each; merged back and forth
    uint32_t* order[2];  // and the tokens' positions
    float* partials;     // two rows of dim floats per kSumChunk sorted tokens
};

// table[v] = scale * the sum of grad[t] over the t with ids[t] == v, in
// ascending t (accumulate: added to table[v], rows without a token untouched;
// else every row is written).  Ids outside [0, vocab) and `padding` have no
// part.
hipError_t launch_lookup_grad(const Rows& grad, int64_t tokens, const TokenIds& ids, int64_t padding, float scale,
                              bool accumulate, const Rows& table, int64_t vocab, int32_t dim,
                              const LookupGradScratch& scratch, hipStream_t stream);

}  // namespace micro

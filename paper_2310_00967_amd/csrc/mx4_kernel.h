// Launches of the microscaled 4-bit calls (mx4_kernel.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "lookup_kernel.h"

namespace micro {

// Values of a block, which share a scale, and of a group, whose codes and scales
// lie beside those of the next row: a step of the products reads whole lines of a
// tile's rows, whatever the rows' length.
constexpr int kMxBlock = 32, kMxGroup = 128, kMxBlocks = kMxGroup / kMxBlock, kMxBytes = kMxGroup / 2;

struct Mx4 {
    char* codes;      // [groups][rows][kMxBytes]
    uint8_t* scales;  // [groups][rows][kMxBlocks]
    int64_t rows, cols, groups;
};

// packed, turned: codes NULL where not wanted.
hipError_t launch_mx4_pack(const Rows& x, int64_t rows, int64_t cols, const Mx4& packed, const Mx4& turned,
                           hipStream_t stream);
hipError_t launch_mx4_unpack(const Mx4& packed, const Rows& out, hipStream_t stream);

// out[i][j] (+)= sum over k of a[i][k] b[j][k].
struct Mx4Product {
    Mx4 a, b;
    Rows out;
    bool accumulate;
    int compute_units;
    float* parts;  // scratch: the parts of tiles whose sums are cut, kMxParts floats a compute unit
};
constexpr int64_t kMxParts = 256 * 256;
hipError_t launch_mx4_product(const Mx4Product& call, hipStream_t stream);
// The same of x, whose packed form goes into call.a if anywhere.
hipError_t launch_mx4_linear(const Rows& x, const Mx4Product& call, hipStream_t stream);

}  // namespace micro

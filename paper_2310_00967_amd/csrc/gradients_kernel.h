// Launches of the gradient set's kernels (gradients_kernel.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace micro {

// A run of consecutive values of one tensor, the unit that a workgroup takes.
struct GradPiece {
    void* values;     // device address of its first value
    int64_t offset;   // of that value in the flat vector
    int32_t count;    // at most GradSetDevice::piece
    int32_t type;     // MICRO_TYPE_*
};

constexpr int kGradBlock = 256;
// Workgroups of a pass at most, and so partial sums.
constexpr int kGradGridMax = 2048;

struct GradSetDevice {
    const GradPiece* pieces;
    int64_t count;         // pieces
    int64_t total;         // values
    double* partials;      // one per workgroup, kGradGridMax
};

// The workgroups' sums of squares into the partials.
hipError_t launch_grads_sums(const GradSetDevice& set, hipStream_t stream);

// *sumsq = the sum of the squares of every value; *norm = its root (either
// may be null).
hipError_t launch_grads_norm(const GradSetDevice& set, double* sumsq, float* norm, hipStream_t stream);

// Every value times min(1, max_norm / (sqrt(squares) + 1e-6)) (scaled false:
// times 1), in place (flat null) or into flat, with squares = *sumsq, or where
// that is null what launch_grads_sums left; *norm = sqrt(squares) unless null.
hipError_t launch_grads_scale(const GradSetDevice& set, bool scaled, const double* sumsq, double max_norm, float* flat,
                              float* norm, hipStream_t stream);

}  // namespace micro

// gfx950 kernels of a gradient set: the global norm over many tensors, and
// their clipping in place or into the flat vector that the sparsify step
// reads.
//   norm    sum of squares, each product and every addition in binary64 (the
//           product of two binary32 values is exact there);
//   factor  c = min(1, max_norm / (norm + 1e-6)) in binary64, once rounded to
//           binary32; a norm of +inf gives 0, a NaN gives NaN;
//   scale   c * g in binary32, once rounded to the destination's type.
// Both are streams, bound by HBM: the norm reads every value once, the scale
// reads it again (no value can be scaled before the last is summed) and
// writes it.  Tensors are cut into pieces of equal length on the host, so one
// launch covers all of them and a workgroup's work does not depend on how a
// model is cut into tensors.  292 bfloat16 tensors of 1.32G values: norm 2.6 GB
// in 425 us (6.2 TB/s), scale into the flat vector 7.9 GB in 1510 us (5.2 TB/s).
#include "gradients_kernel.h"
#include "launch.h"
#include "micro_sparsify.h"
#include "value_types.h"

namespace micro {
namespace {

// Loads that a thread has in flight before it uses the first.  Two, four and
// one are within a percent of each other; eight spill the occupancy that hides
// the rest (the norm of 11.7M values alone then takes as long as both passes).
constexpr int kUnroll = 2;

template <class T>
__device__ double sum_squares(const T* p, int n) {
    constexpr int kVec = 16 / sizeof(T), kStep = kGradBlock * kVec;
    double sum[kUnroll] = {};
    int i = threadIdx.x * kVec;
    for (; i + (kUnroll - 1) * kStep + kVec <= n; i += kUnroll * kStep) {
        float x[kUnroll][kVec];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) load_floats<T, kVec>(p + i + u * kStep, x[u]);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int j = 0; j < kVec; ++j) {
                const double d = static_cast<double>(x[u][j]);
                sum[u] = __builtin_fma(d, d, sum[u]);
            }
    }
    for (; i < n; i += kStep)
        for (int j = i; j < n && j < i + kVec; ++j) {
            const double d = static_cast<double>(static_cast<float>(p[j]));
            sum[0] = __builtin_fma(d, d, sum[0]);
        }
#pragma unroll
    for (int u = 1; u < kUnroll; ++u) sum[0] += sum[u];
    return sum[0];
}

// The sum over the workgroup, in a fixed order; in thread 0.
__device__ double block_sum(double x) {
    __shared__ double waves[kGradBlock / 64];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
    __syncthreads();
    double sum = 0.0;
    for (int w = 0; w < kGradBlock / 64; ++w) sum += waves[w];
    return sum;
}

// A workgroup takes every gridDim.x-th piece and leaves its sum.
__global__ __launch_bounds__(kGradBlock) void norm_kernel(GradSetDevice set) {
    double sum = 0.0;
    for (int64_t i = blockIdx.x; i < set.count; i += gridDim.x) {
        const GradPiece piece = set.pieces[i];
        if (piece.type == MICRO_TYPE_F32)
            sum += sum_squares(static_cast<const float*>(piece.values), piece.count);
        else if (piece.type == MICRO_TYPE_F16)
            sum += sum_squares(static_cast<const f16*>(piece.values), piece.count);
        else
            sum += sum_squares(static_cast<const bf16*>(piece.values), piece.count);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) set.partials[blockIdx.x] = sum;
}

// The sum of the workgroups' sums, in their order: the same in every thread of
// every workgroup that asks.  `count` of them, kGradGridMax at most.
__device__ double add_partials(const double* partials, int count) {
    constexpr int kEach = kGradGridMax / kGradBlock;
    double x[kEach], sum = 0.0;
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int i = threadIdx.x + u * kGradBlock;
        x[u] = partials[i < count ? i : 0];
    }
#pragma unroll
    for (int u = 0; u < kEach; ++u) sum += static_cast<int>(threadIdx.x + u * kGradBlock) < count ? x[u] : 0.0;
    return block_sum(sum);
}

__global__ __launch_bounds__(kGradBlock) void total_kernel(const double* partials, int count, double* sumsq, float* norm) {
    const double sum = add_partials(partials, count);
    if (threadIdx.x != 0) return;
    if (sumsq) *sumsq = sum;
    if (norm) *norm = static_cast<float>(sqrt(sum));
}

// n values of src times c into dst, which may be src.
template <bool kPast, class S, class D>
__device__ void scale_run(const S* src, D* dst, int n, float c) {
    // as many values a thread as make the wider side's access 16 bytes
    constexpr int kVec = 16 / (sizeof(S) > sizeof(D) ? sizeof(S) : sizeof(D)), kStep = kGradBlock * kVec;
    int i = threadIdx.x * kVec;
    for (; i + (kUnroll - 1) * kStep + kVec <= n; i += kUnroll * kStep) {
        float x[kUnroll][kVec];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) load_floats<S, kVec>(src + i + u * kStep, x[u]);
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
            for (int j = 0; j < kVec; ++j) x[u][j] *= c;
            if constexpr (kPast)
                stream_floats<D, kVec>(dst + i + u * kStep, x[u]);
            else
                store_floats<D, kVec>(dst + i + u * kStep, x[u]);
        }
    }
    for (; i < n; i += kStep)
        for (int j = i; j < n && j < i + kVec; ++j) dst[j] = rounded<D>(static_cast<float>(src[j]) * c);
}

template <class T>
__device__ void scale_piece(const GradPiece& piece, float* flat, bool past, float c) {
    T* values = static_cast<T*>(piece.values);
    if (!flat)
        scale_run<false, T, T>(values, values, piece.count, c);
    else if (past)
        scale_run<true, T, float>(values, flat + piece.offset, piece.count, c);
    else
        scale_run<false, T, float>(values, flat + piece.offset, piece.count, c);
}

// scaled: whether c is not simply 1.  The squared norm is *sumsq, or where that
// is null the sum of the `sums` partial ones, which every workgroup adds for
// itself: a microsecond, where one workgroup's adding and its signal to the
// others take several.  The pieces are taken last to first: those that the norm
// read last are still in the cache.  past: the flat vector is larger than that
// cache.  On 335M values (671 MB of bf16) the order and the stores past the
// cache took the two passes from 524 to 483 us.
__global__ __launch_bounds__(kGradBlock) void scale_kernel(GradSetDevice set, bool scaled, const double* sumsq, int sums,
                                                           double max_norm, float* flat, bool past, float* norm) {
    float c = 1.0f;
    if (scaled) {
        const double length = sqrt(sumsq ? *sumsq : add_partials(set.partials, sums)), ratio = max_norm / (length + 1e-6);
        if (max_norm < __builtin_inf() && !(ratio >= 1.0)) c = static_cast<float>(ratio);
        if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = static_cast<float>(length);
    }
    if (!flat && c == 1.0f) return;  // in place and nothing to clip
    for (int64_t i = set.count - 1 - blockIdx.x; i >= 0; i -= gridDim.x) {
        const GradPiece piece = set.pieces[i];
        if (piece.type == MICRO_TYPE_F32)
            scale_piece<float>(piece, flat, past, c);
        else if (piece.type == MICRO_TYPE_F16)
            scale_piece<f16>(piece, flat, past, c);
        else
            scale_piece<bf16>(piece, flat, past, c);
    }
}

// The memory-side cache.
constexpr int64_t kCacheBytes = int64_t(256) << 20;

int pass_grid(int64_t pieces) {
    return static_cast<int>(pieces < 1 ? 1 : pieces > kGradGridMax ? kGradGridMax : pieces);
}

}  // namespace

hipError_t launch_grads_sums(const GradSetDevice& set, hipStream_t stream) {
    return launch(norm_kernel, dim3(pass_grid(set.count)), dim3(kGradBlock), stream, set);
}

hipError_t launch_grads_norm(const GradSetDevice& set, double* sumsq, float* norm, hipStream_t stream) {
    const hipError_t e = launch_grads_sums(set, stream);
    if (e != hipSuccess) return e;
    return launch(total_kernel, dim3(1), dim3(kGradBlock), stream, set.partials, pass_grid(set.count), sumsq, norm);
}

hipError_t launch_grads_scale(const GradSetDevice& set, bool scaled, const double* sumsq, double max_norm, float* flat,
                              float* norm, hipStream_t stream) {
    return launch(scale_kernel, dim3(pass_grid(set.count)), dim3(kGradBlock), stream, set, scaled, sumsq,
                  pass_grid(set.count), max_norm, flat, set.total * 4 > kCacheBytes, norm);
}

}  // namespace micro

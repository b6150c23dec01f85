// gfx950 kernels of microscaled 4-bit matrices: blocks of 32 values with a power
// of two as their scale,
//   e = floor(log2 max |v|) - 2,   code = v / 2^e to the nearest of
//   +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}, ties to the even code,
// and the product of two such matrices by the matrix cores' scaled instruction,
// which multiplies codes and both scales exactly and sums in binary32.
#include "mx4_kernel.h"

#include <algorithm>

#include "launch.h"
#include "micro_sparsify.h"
#include "value_types.h"

namespace micro {
namespace {

using Words4 = int __attribute__((ext_vector_type(4)));
using Words8 = int __attribute__((ext_vector_type(8)));
using Acc = float __attribute__((ext_vector_type(16)));

// What the two scales of a 32 x 32 x 64 product come from: the bytes of a word
// for each lane's row, one of which (step) it takes.
__device__ __forceinline__ Words8 half_of(Words4 x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }
constexpr int kFp4 = 4;
template <int kStep>
__device__ __forceinline__ Acc mma(Words4 a, uint32_t sa, Words4 b, uint32_t sb, Acc c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(half_of(a), half_of(b), c, kFp4, kFp4, kStep,
                                                           static_cast<int>(sa), kStep, static_cast<int>(sb));
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

constexpr uint32_t kNanScale = 255;

// The scale byte of a block whose largest magnitude has these bits: the exponent
// field of 2^(floor(log2 a) - 2); subnormal magnitudes have field 0 and end at
// the least scale, 2^-127, as zeros do.
__device__ __forceinline__ uint32_t scale_of(uint32_t most) {
    const uint32_t field = most >> 23;
    return field == 255 ? kNanScale : field > 2 ? field - 2 : 0;
}
// 2^-e, by which the block's values are multiplied; a NaN block's become codes 0.
__device__ __forceinline__ float inverse_of(uint32_t scale) { return __uint_as_float((254 - scale) << 23); }
__device__ __forceinline__ float power_of(uint32_t scale) {
    return scale == kNanScale ? __builtin_nanf("") : scale == 0 ? 0x1p-127f : __uint_as_float(scale << 23);
}

// Eight codes, the first in the lowest bits.  The conversion rounds to nearest
// even and ends at 6.
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], uint32_t scale) {
    if (scale == kNanScale) return 0;
    const float by = inverse_of(scale);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0] * by, v[1] * by, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2] * by, v[3] * by, 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4] * by, v[5] * by, 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6] * by, v[7] * by, 1.0f, 3);
    return c;
}

// ---------------------------------------------------------------------------
// packing
// ---------------------------------------------------------------------------

template <class T, int N>
__device__ __forceinline__ void load_some(const T* p, int64_t valid, float (&v)[N]) {
    if (valid >= N) {
        load_floats(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < valid ? static_cast<float>(p[i]) : 0.0f;
    }
}

// Rows: a workgroup takes kPackRows rows of kPackGroups groups, half a wavefront
// a row's group, eight values a lane.
constexpr int kPackThreads = 256, kPackRows = 16, kPackGroups = 4;
template <class T>
__global__ __launch_bounds__(kPackThreads) void pack_kernel(const T* x, int64_t stride, Mx4 to) {
    const int64_t wide = (to.groups + kPackGroups - 1) / kPackGroups;
    const int64_t tiles = (to.rows + kPackRows - 1) / kPackRows * wide;
    const int lane = threadIdx.x & 31, half = threadIdx.x >> 5;
    constexpr int kRowsAtOnce = kPackThreads / 32 / kPackGroups;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t g = tile % wide * kPackGroups + half % kPackGroups;
        const int64_t r0 = tile / wide * kPackRows + half / kPackGroups;
        if (g >= to.groups) continue;
        const int64_t c = g * kMxGroup + lane * 8;
#pragma unroll
        for (int i = 0; i < kPackRows / kRowsAtOnce; ++i) {
            const int64_t r = r0 + i * kRowsAtOnce;
            if (r >= to.rows) break;
            float v[8];
            load_some(x + r * stride + c, to.cols - c, v);
            uint32_t most = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) most = max(most, magnitude(v[j]));
            most = max(most, __shfl_xor(most, 1));
            most = max(most, __shfl_xor(most, 2));
            const uint32_t scale = scale_of(most);
            *reinterpret_cast<uint32_t*>(to.codes + (r * to.groups + g) * kMxLine + lane * 4) = codes_of(v, scale);
            if ((lane & 3) == 0) to.scales[(g * to.rows + r) * 8 + lane / 4] = static_cast<uint8_t>(scale);
        }
    }
}

// Columns: a thread takes kVec adjacent columns of one block of 32 rows, the
// eight blocks of a group beside each other, so a column's line of codes is
// written by eight lanes.
template <class T>
__global__ __launch_bounds__(kPackThreads) void pack_turned_kernel(const T* x, int64_t stride, Mx4 to) {
    constexpr int kVec = 16 / sizeof(T), kColumns = 8 * kVec * kPackThreads / 64;
    const int64_t across = (to.rows + kColumns - 1) / kColumns, tiles = across * to.groups;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, block = lane >> 3;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t g = tile / across;
        const int64_t c = tile % across * kColumns + (wave * 8 + (lane & 7)) * kVec;
        const int64_t k = g * kMxGroup + block * kMxBlock;
        if (c >= to.rows) continue;
        float v[kMxBlock][kVec];
#pragma unroll
        for (int i = 0; i < kMxBlock; ++i) load_some(x + (k + i) * stride + c, k + i < to.cols ? to.rows - c : 0, v[i]);
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            if (c + j >= to.rows) break;
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < kMxBlock; ++i) most = max(most, magnitude(v[i][j]));
            const uint32_t scale = scale_of(most);
            Words4 codes;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = v[q * 8 + i][j];
                codes[q] = static_cast<int>(codes_of(w, scale));
            }
            *reinterpret_cast<Words4*>(to.codes + ((c + j) * to.groups + g) * kMxLine + block * 16) = codes;
            to.scales[(g * to.rows + c + j) * 8 + block] = static_cast<uint8_t>(scale);
        }
    }
}

template <class T>
__global__ __launch_bounds__(kPackThreads) void unpack_kernel(Mx4 from, T* out, int64_t stride) {
    const int64_t lines = from.rows * from.groups;
    const int lane = threadIdx.x & 31;
    for (int64_t line = static_cast<int64_t>(blockIdx.x) * (kPackThreads / 32) + (threadIdx.x >> 5); line < lines;
         line += static_cast<int64_t>(gridDim.x) * (kPackThreads / 32)) {
        const int64_t r = line / from.groups, g = line - r * from.groups, c = g * kMxGroup + lane * 8;
        if (c >= from.cols) continue;
        const uint32_t codes = *reinterpret_cast<const uint32_t*>(from.codes + line * kMxLine + lane * 4);
        const float by = power_of(from.scales[(g * from.rows + r) * 8 + lane / 4]);
        float v[8];
        const auto two = [&](auto pair, int i) {
            v[i] = pair[0] * by;
            v[i + 1] = pair[1] * by;
        };
        two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0), 0);
        two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1), 2);
        two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2), 4);
        two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3), 6);
        T* p = out + r * stride + c;
        if (c + 8 <= from.cols) {
            store_floats(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < from.cols) p[i] = rounded<T>(v[i]);
        }
    }
}

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------

// Where a lane's operand comes from: row `row` of a matrix, clamped to its last;
// half 0 of a wavefront takes the first four blocks of a group, half 1 the others
// (a sum's order is free, and both operands agree).
struct Side {
    const char* codes;
    const uint8_t* scales;
    int64_t scale_step;
    __device__ Side(const Mx4& m, int64_t row, int half) {
        const int64_t r = row < m.rows ? row : m.rows - 1;
        codes = m.codes + r * m.groups * kMxLine + half * 64;
        scales = m.scales + r * 8 + half * 4;
        scale_step = m.rows * 8;
    }
    __device__ __forceinline__ void load(int64_t g, Words4 (&c)[4], uint32_t& s) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = *reinterpret_cast<const Words4*>(codes + g * kMxLine + i * 16);
        s = *reinterpret_cast<const uint32_t*>(scales + g * scale_step);
    }
};

// A tile of 32 x 32 a workgroup, whose four wavefronts take every fourth group
// and add their sums in shared memory.
constexpr int kTile = 32, kFewWaves = 4, kPadded = kTile + 4;
template <class T>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(Mx4 a, Mx4 b, T* out, int64_t stride, bool accumulate) {
    __shared__ __attribute__((aligned(16))) float sums[kFewWaves][kTile][kPadded];
    const int64_t down = (a.rows + kTile - 1) / kTile, tiles = down * ((b.rows + kTile - 1) / kTile);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t i0 = tile % down * kTile, j0 = tile / down * kTile;
        const Side sa(a, i0 + (lane & 31), half), sb(b, j0 + (lane & 31), half);
        Acc acc;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
        for (int64_t g = wave; g < a.groups; g += kFewWaves) {
            Words4 ca[4], cb[4];
            uint32_t xa, xb;
            sb.load(g, cb, xb);
            sa.load(g, ca, xa);
            acc = mma<0>(cb[0], xb, ca[0], xa, acc);
            acc = mma<1>(cb[1], xb, ca[1], xa, acc);
            acc = mma<2>(cb[2], xb, ca[2], xa, acc);
            acc = mma<3>(cb[3], xb, ca[3], xa, acc);
        }
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<float4*>(&sums[wave][lane & 31][q * 8 + half * 4]) =
                make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
        __syncthreads();
        const int64_t i = i0 + threadIdx.x / 8, j = j0 + threadIdx.x % 8 * 4;
        if (i >= a.rows || j >= b.rows) continue;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] += sums[w][threadIdx.x / 8][threadIdx.x % 8 * 4 + q];
        T* p = out + i * stride + j;
        if (j + 4 <= b.rows) {
            if (accumulate) {
                float old[4];
                load_floats(p, old);
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] += old[q];
            }
            store_floats(p, v);
        } else {
            for (int q = 0; q < 4; ++q)
                if (j + q < b.rows) p[q] = rounded<T>(accumulate ? v[q] + static_cast<float>(p[q]) : v[q]);
        }
    }
}

constexpr int64_t kMostGroups = int64_t(1) << 20;
dim3 grid_of(int64_t n) { return dim3(static_cast<uint32_t>(std::min(n, kMostGroups))); }

template <class T>
hipError_t pack(const Rows& x, const Mx4& packed, const Mx4& turned, hipStream_t stream) {
    const T* at = static_cast<const T*>(x.at);
    if (packed.codes)
        if (const hipError_t e = launch(pack_kernel<T>,
                                        grid_of((packed.rows + kPackRows - 1) / kPackRows *
                                                ((packed.groups + kPackGroups - 1) / kPackGroups)),
                                        kPackThreads, stream, at, x.stride, packed))
            return e;
    if (!turned.codes) return hipSuccess;
    constexpr int kColumns = 8 * (16 / sizeof(T)) * kPackThreads / 64;
    return launch(pack_turned_kernel<T>, grid_of((turned.rows + kColumns - 1) / kColumns * turned.groups), kPackThreads,
                  stream, at, x.stride, turned);
}

}  // namespace

hipError_t launch_mx4_pack(const Rows& x, int64_t rows, int64_t cols, const Mx4& packed, const Mx4& turned,
                           hipStream_t stream) {
    if (rows == 0 || cols == 0) return hipSuccess;
    switch (x.type) {
        case MICRO_TYPE_F32: return pack<float>(x, packed, turned, stream);
        case MICRO_TYPE_F16: return pack<f16>(x, packed, turned, stream);
        default: return pack<bf16>(x, packed, turned, stream);
    }
}

hipError_t launch_mx4_unpack(const Mx4& from, const Rows& out, hipStream_t stream) {
    if (from.rows == 0 || from.cols == 0) return hipSuccess;
    const dim3 grid = grid_of((from.rows * from.groups + kPackThreads / 32 - 1) / (kPackThreads / 32));
    switch (out.type) {
        case MICRO_TYPE_F32:
            return launch(unpack_kernel<float>, grid, kPackThreads, stream, from, static_cast<float*>(out.at), out.stride);
        case MICRO_TYPE_F16:
            return launch(unpack_kernel<f16>, grid, kPackThreads, stream, from, static_cast<f16*>(out.at), out.stride);
        default:
            return launch(unpack_kernel<bf16>, grid, kPackThreads, stream, from, static_cast<bf16*>(out.at), out.stride);
    }
}

namespace {

template <class T>
hipError_t product(const Mx4Product& c, hipStream_t stream) {
    const int64_t tiles = (c.a.rows + kTile - 1) / kTile * ((c.b.rows + kTile - 1) / kTile);
    return launch(few_kernel<T>, grid_of(tiles), 64 * kFewWaves, stream, c.a, c.b, static_cast<T*>(c.out.at), c.out.stride,
                  c.accumulate);
}

}  // namespace

hipError_t launch_mx4_product(const Mx4Product& c, hipStream_t stream) {
    if (c.a.rows == 0 || c.b.rows == 0) return hipSuccess;
    switch (c.out.type) {
        case MICRO_TYPE_F32: return product<float>(c, stream);
        case MICRO_TYPE_F16: return product<f16>(c, stream);
        default: return product<bf16>(c, stream);
    }
}

}  // namespace micro

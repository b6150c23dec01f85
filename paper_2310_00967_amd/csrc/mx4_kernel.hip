// gfx950 kernels of microscaled 4-bit matrices: blocks of 32 values with a power
// of two as their scale,
//   e = floor(log2 max |v|) - 2,   code = v / 2^e to the nearest of
//   +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}, ties to the even code,
// and the product of two such matrices by the matrix cores' scaled instruction,
// which multiplies codes and both scales exactly and sums in binary32.
#include "mx4_kernel.h"

#include <algorithm>
#include <type_traits>

#include "launch.h"
#include "micro_sparsify.h"
#include "product_tiles.h"
#include "value_types.h"

namespace micro {
namespace {

using Words4 = int __attribute__((ext_vector_type(4)));
using Words8 = int __attribute__((ext_vector_type(8)));

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

// Codes of kN values, the first in the lowest bits.  The conversion rounds to nearest
// even and ends at 6.
template <int kN>
__device__ __forceinline__ uint32_t codes_of(const float (&v)[kN], uint32_t scale) {
    static_assert(kN == 4 || kN == 8, "two values a byte");
    if (scale == kNanScale) return 0;
    const float by = inverse_of(scale);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0] * by, v[1] * by, 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2] * by, v[3] * by, 1.0f, 1);
    if constexpr (kN == 8) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4] * by, v[5] * by, 1.0f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6] * by, v[7] * by, 1.0f, 3);
    }
    return c;
}

// The largest of this lane's value and others': of the four lanes of its quad, of the
// quad beside it.
template <int kControl>
__device__ __forceinline__ uint32_t most_with(uint32_t x) {
    return max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0u, x, kControl, 0xf, 0xf, false)));
}
__device__ __forceinline__ uint32_t most_of_quad(uint32_t x) { return most_with<0x4e>(most_with<0xb1>(x)); }
__device__ __forceinline__ uint32_t most_of_eight(uint32_t x) { return most_with<0x141>(most_of_quad(x)); }

// ---------------------------------------------------------------------------
// packing
// ---------------------------------------------------------------------------

// N values of which the first `valid` are there, zeros behind.
template <class T, int N>
__device__ __forceinline__ Pack<T, N> load_some(const T* p, int64_t valid) {
    if (valid >= N) return *reinterpret_cast<const Pack<T, N>*>(p);
    Pack<T, N> v;
#pragma unroll
    for (int i = 0; i < N; ++i) v.v[i] = i < valid ? p[i] : static_cast<T>(0.0f);
    return v;
}

// Rows: a workgroup takes kPackRows rows of kPackGroups groups, sixteen lanes a row's
// group, eight values a lane, so that neighbouring lanes read one row and the
// workgroup's stores fill whole lines of a group's rows.  Bound by memory: 50257 x 2048
// bfloat16 values in 49 to 57 us, 4.6 to 5.4 TB/s.
constexpr int kPackThreads = 256, kPackRows = 8, kPackGroups = 8, kPackLanes = kMxGroup / 8;
template <class T>
__global__ __launch_bounds__(kPackThreads) void pack_kernel(const T* x, int64_t stride, Mx4 to) {
    const int lane = threadIdx.x % kPackLanes, part = threadIdx.x / kPackLanes;
    constexpr int kRowsAtOnce = kPackThreads / kPackLanes / kPackGroups;
    const int64_t g = static_cast<int64_t>(blockIdx.x) * kPackGroups + part / kRowsAtOnce;
    const int64_t c = g * kMxGroup + lane * 8;
    if (g >= to.groups) return;
    for (int64_t r0 = static_cast<int64_t>(blockIdx.y) * kPackRows + part % kRowsAtOnce; r0 < to.rows;
         r0 += static_cast<int64_t>(gridDim.y) * kPackRows) {
        constexpr int kEach = kPackRows / kRowsAtOnce;
        Pack<T, 8> raw[kEach];
        if (c + 8 <= to.cols && r0 + (kEach - 1) * kRowsAtOnce < to.rows) {  // the loads go out together
#pragma unroll
            for (int i = 0; i < kEach; ++i) raw[i] = *reinterpret_cast<const Pack<T, 8>*>(x + (r0 + i * kRowsAtOnce) * stride + c);
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int64_t r = r0 + i * kRowsAtOnce;
                raw[i] = load_some<T, 8>(x + r * stride + c, r < to.rows ? to.cols - c : 0);
            }
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int64_t r = r0 + i * kRowsAtOnce;
            if (r >= to.rows) break;
            float v[8];
            uint32_t most = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = static_cast<float>(raw[i].v[j]);
                most = max(most, magnitude(v[j]));
            }
            const uint32_t scale = scale_of(most_of_quad(most));
            *reinterpret_cast<uint32_t*>(to.codes + (g * to.rows + r) * kMxBytes + lane * 4) = codes_of(v, scale);
            if ((lane & 3) == 0) to.scales[(g * to.rows + r) * kMxBlocks + lane / 4] = static_cast<uint8_t>(scale);
        }
    }
}

// Columns, and rows from the same reading: a workgroup takes a group of kMxGroup rows by
// kTurnColumns columns, a thread kTurnVec adjacent columns of one block of 32 rows in
// registers.  The four blocks of a group lie beside each other, so that the turned codes
// of neighbouring columns are written as whole lines; those of the rows change places in
// shared memory, to leave as runs of kMxGroup rows of a group.
// Four columns a thread: with eight, of 16-bit types, the values take 256 registers and
// 16384 x 8192 takes 180 us for 69 (rows alone 65, both ways 90 to 108).
constexpr int kTurnVec = 4, kTurnColumns = 64 / kMxBlocks * kTurnVec * (kPackThreads / 64);
static_assert(kTurnColumns == 2 * kMxGroup, "two groups of rows' values");
template <class T, bool kRows>
__global__ __launch_bounds__(kPackThreads) void pack_turned_kernel(const T* x, int64_t stride, Mx4 rows, Mx4 turned) {
    __shared__ __attribute__((aligned(16))) uint16_t codes[kRows ? 2 : 1][kRows ? kMxGroup : 1][kMxBytes / 2];
    __shared__ __attribute__((aligned(16))) uint8_t scales[kRows ? 2 : 1][kRows ? kMxGroup : 1][kMxBlocks];
    constexpr int kAcross = 64 / kMxBlocks;  // threads of a wavefront along a row
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, block = lane / kAcross;
    const int at = (wave * kAcross + lane % kAcross) * kTurnVec;  // in the workgroup's columns
    const int64_t c0 = static_cast<int64_t>(blockIdx.x) * kTurnColumns, c = c0 + at;
    for (int64_t g = blockIdx.y; g < turned.groups; g += gridDim.y) {
        const int64_t k = g * kMxGroup + block * kMxBlock;
        Pack<T, kTurnVec> raw[kMxBlock];
        if (turned.rows % kTurnVec == 0) {
            // from the nearest place in x, all at once; what lies outside is 0
            const T* from = x + (c < turned.rows ? c : turned.rows - kTurnVec);
#pragma unroll
            for (int i = 0; i < kMxBlock; ++i)
                raw[i] = *reinterpret_cast<const Pack<T, kTurnVec>*>(from + (k + i < turned.cols ? k + i : turned.cols - 1) * stride);
            if (c0 + kTurnColumns > turned.rows || (g + 1) * kMxGroup > turned.cols)
#pragma unroll
                for (int i = 0; i < kMxBlock; ++i)
                    if (c >= turned.rows || k + i >= turned.cols) raw[i] = Pack<T, kTurnVec>{};
        } else {
#pragma unroll
            for (int i = 0; i < kMxBlock; ++i)
                raw[i] = load_some<T, kTurnVec>(x + (k + i) * stride + c, k + i < turned.cols ? turned.rows - c : 0);
        }
        const auto value = [&](int i, int j) { return static_cast<float>(raw[i].v[j]); };
#pragma unroll
        for (int j = 0; j < kTurnVec; ++j) {
            if (c + j >= turned.rows) break;
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < kMxBlock; ++i) most = max(most, magnitude(value(i, j)));
            const uint32_t scale = scale_of(most);
            Words4 q;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                float y[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = value(w * 8 + i, j);
                q[w] = static_cast<int>(codes_of(y, scale));
            }
            *reinterpret_cast<Words4*>(turned.codes + (g * turned.rows + c + j) * kMxBytes + block * 16) = q;
            turned.scales[(g * turned.rows + c + j) * kMxBlocks + block] = static_cast<uint8_t>(scale);
        }
        if constexpr (kRows) {
            const int half = at / kMxGroup, byte = at % kMxGroup / 2;
#pragma unroll
            for (int i = 0; i < kMxBlock; ++i) {
                uint32_t most = 0;
                float y[kTurnVec];
#pragma unroll
                for (int j = 0; j < kTurnVec; ++j) {
                    y[j] = value(i, j);
                    most = max(most, magnitude(y[j]));
                }
                const uint32_t scale = scale_of(most_of_eight(most));
                codes[half][block * kMxBlock + i][byte / 2] = static_cast<uint16_t>(codes_of(y, scale));
                if ((lane & 7) == 0) scales[half][block * kMxBlock + i][byte / 16] = static_cast<uint8_t>(scale);
            }
            __syncthreads();
            const int64_t left = rows.rows - g * kMxGroup;
            const int count = left < kMxGroup ? static_cast<int>(left) : kMxGroup;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t of = c0 / kMxGroup + h;
                if (of >= rows.groups) break;
                const int64_t first = of * rows.rows + g * kMxGroup;
                for (int i = threadIdx.x; i < count * kMxBytes / 16; i += kPackThreads)
                    reinterpret_cast<Words4*>(rows.codes + first * kMxBytes)[i] = reinterpret_cast<const Words4*>(codes[h])[i];
                if (static_cast<int>(threadIdx.x) < count)
                    reinterpret_cast<uint32_t*>(rows.scales + first * kMxBlocks)[threadIdx.x] =
                        reinterpret_cast<const uint32_t*>(scales[h])[threadIdx.x];
            }
            __syncthreads();
        }
    }
}

// The way back: sixteen lanes a row's group as above, each 16 bytes of out at a time, a row
// after the other, so that workgroups in their order write memory in its order: 50257 x
// 2048 bfloat16 values in 55 to 58 us (4.5 to 4.7 TB/s; 73 where each call writes other
// memory), by workgroups of 8 rows and 8 groups in 68.
template <class T>
__global__ __launch_bounds__(kPackThreads) void unpack_kernel(Mx4 from, T* out, int64_t stride) {
    constexpr int kVec = 16 / sizeof(T), kPieces = 8 / kVec, kLines = kPackThreads / kPackLanes;
    using Codes = typename std::conditional<kVec == 8, uint32_t, uint16_t>::type;
    const int64_t lines = from.rows * from.groups;
    const int lane = threadIdx.x % kPackLanes;
    for (int64_t line = static_cast<int64_t>(blockIdx.x) * kLines + threadIdx.x / kPackLanes; line < lines;
         line += static_cast<int64_t>(gridDim.x) * kLines) {
        const int64_t r = lines < int64_t(1) << 32 ? static_cast<uint32_t>(line) / static_cast<uint32_t>(from.groups)
                                                   : line / from.groups;
        const int64_t g = line - r * from.groups;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int at = p * (kPackLanes * kVec) + lane * kVec;  // in the group
            const int64_t c = g * kMxGroup + at;
            if (c >= from.cols) break;
            const uint32_t codes = *reinterpret_cast<const Codes*>(from.codes + (g * from.rows + r) * kMxBytes + at / 2);
            const float by = power_of(from.scales[(g * from.rows + r) * kMxBlocks + at / kMxBlock]);
            float v[kVec];
            const auto two = [&](auto pair, int i) {
                v[i] = pair[0] * by;
                v[i + 1] = pair[1] * by;
            };
            two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0), 0);
            two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1), 2);
            if constexpr (kVec == 8) {
                two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2), 4);
                two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3), 6);
            }
            T* to = out + r * stride + c;
            if (c + kVec <= from.cols) {
                store_floats(to, v);
            } else {
#pragma unroll
                for (int j = 0; j < kVec; ++j)
                    if (c + j < from.cols) to[j] = rounded<T>(v[j]);
            }
        }
    }
}

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------

// Where a lane's operand comes from: row `row` of a matrix, clamped to its last;
// half 0 of a wavefront takes the first two blocks of a group, half 1 the others
// (a sum's order is free, and both operands agree).
struct Side {
    const char* codes;
    const uint8_t* scales;
    int64_t rows;
    __device__ Side(const Mx4& m, int64_t row, int half) : rows(m.rows) {
        const int64_t r = row < m.rows ? row : m.rows - 1;
        codes = m.codes + r * kMxBytes + half * 32;
        scales = m.scales + r * kMxBlocks + half * 2;
    }
    __device__ __forceinline__ void load(int64_t g, Words4 (&c)[2], uint32_t& s) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) c[i] = *reinterpret_cast<const Words4*>(codes + g * rows * kMxBytes + i * 16);
        s = *reinterpret_cast<const uint16_t*>(scales + g * rows * kMxBlocks);
    }
};

// A tile of 32 x 32 a workgroup, whose four wavefronts take every fourth group, two at a
// time, and add their sums in shared memory.  Bound by one read of b: 1 x 2048 x 50257 in
// 13.8 us (4.0 TB/s of 55 MB from memory), 32 rows in 18.2; one group at a time 14.6 and
// 21.5, four 14.0 and 17.6 but 7.5 for 6.2 at 1 x 1024 x 30522.  (Sizes of products are
// rows x length of the sums x columns, here and below.)
constexpr int kTile = 32, kFewWaves = 4, kFewAhead = 2, kPadded = kTile + 4;
struct FewOut {
    void* at;
    int64_t stride, rows, columns;
    bool accumulate;
};
using FewSums = float[kFewWaves][kTile][kPadded];

template <class T>
__device__ __forceinline__ void finish_few(FewSums& sums, const Acc& acc, const FewOut& out, int64_t i0, int64_t j0) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(&sums[wave][lane & 31][q * 8 + half * 4]) =
            make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
    __syncthreads();
    const int64_t i = i0 + threadIdx.x / 8, j = j0 + threadIdx.x % 8 * 4;
    if (i >= out.rows || j >= out.columns) return;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += sums[w][threadIdx.x / 8][threadIdx.x % 8 * 4 + q];
    T* p = static_cast<T*>(out.at) + i * out.stride + j;
    if (j + 4 <= out.columns) {
        if (out.accumulate) {
            float old[4];
            load_floats(p, old);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] += old[q];
        }
        store_floats(p, v);
    } else {
        for (int q = 0; q < 4; ++q)
            if (j + q < out.columns) p[q] = rounded<T>(out.accumulate ? v[q] + static_cast<float>(p[q]) : v[q]);
    }
}

template <class T>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(Mx4 a, Mx4 b, FewOut out) {
    __shared__ __attribute__((aligned(16))) FewSums sums;
    const int64_t down = (a.rows + kTile - 1) / kTile, tiles = down * ((b.rows + kTile - 1) / kTile);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t i0 = tile % down * kTile, j0 = tile / down * kTile;
        const Side sa(a, i0 + (lane & 31), half), sb(b, j0 + (lane & 31), half);
        Acc acc;
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
        for (int64_t g = wave; g < a.groups; g += kFewWaves * kFewAhead) {
            Words4 ca[kFewAhead][2], cb[kFewAhead][2];
            uint32_t xa[kFewAhead], xb[kFewAhead];
#pragma unroll
            for (int i = 0; i < kFewAhead; ++i)
                if (g + i * kFewWaves < a.groups) {
                    sb.load(g + i * kFewWaves, cb[i], xb[i]);
                    sa.load(g + i * kFewWaves, ca[i], xa[i]);
                }
#pragma unroll
            for (int i = 0; i < kFewAhead; ++i)
                if (g + i * kFewWaves < a.groups) {
                    acc = mma<0>(cb[i][0], xb[i], ca[i][0], xa[i], acc);
                    acc = mma<1>(cb[i][1], xb[i], ca[i][1], xa[i], acc);
                }
        }
        finish_few<T>(sums, acc, out, i0, j0);
    }
}

// The same for up to 32 rows of x that have kOwnValues values, in whole groups, at most:
// each workgroup packs them for itself, under its first loads of b, which takes less than
// a launch that packs them once (a workgroup's share is 32 values a thread).
constexpr int kOwnValues = 8192;
template <class X, class T>
__global__ __launch_bounds__(64 * kFewWaves) void few_linear_kernel(const X* x, int64_t stride, int rows, Mx4 b, FewOut out) {
    __shared__ __attribute__((aligned(16))) FewSums sums;
    __shared__ __attribute__((aligned(16))) char codes[kOwnValues / 2];
    __shared__ __attribute__((aligned(16))) uint8_t scales[kOwnValues / kMxBlock];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int64_t j0 = static_cast<int64_t>(blockIdx.x) * kTile;
    const int groups = static_cast<int>(b.groups), units = groups * kPackLanes;  // of eight values, of a row
    const Side sb(b, j0 + (lane & 31), half);
    Words4 cb[kFewAhead][2];
    uint32_t xb[kFewAhead];
    const auto load = [&](int g) {
#pragma unroll
        for (int i = 0; i < kFewAhead; ++i)
            if (g + i * kFewWaves < groups) sb.load(g + i * kFewWaves, cb[i], xb[i]);
    };
    load(wave);
    for (int u = threadIdx.x; u < rows * units; u += 64 * kFewWaves) {
        const int r = u / units, c = (u - r * units) * 8;
        const Pack<X, 8> raw = load_some<X, 8>(x + r * stride + c, b.cols - c);
        float v[8];
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = static_cast<float>(raw.v[j]);
            most = max(most, magnitude(v[j]));
        }
        const uint32_t scale = scale_of(most_of_quad(most));
        *reinterpret_cast<uint32_t*>(codes + u * 4) = codes_of(v, scale);
        if ((u & 3) == 0) scales[u / 4] = static_cast<uint8_t>(scale);
    }
    __syncthreads();
    const int row = (lane & 31) < rows ? lane & 31 : rows - 1;
    const char* own = codes + row * groups * kMxBytes + half * 32;
    const uint8_t* own_scales = scales + row * groups * kMxBlocks + half * 2;
    Acc acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
    for (int g = wave; g < groups; g += kFewWaves * kFewAhead) {
        if (g != wave) load(g);
#pragma unroll
        for (int i = 0; i < kFewAhead; ++i) {
            const int of = g + i * kFewWaves;
            if (of >= groups) break;
            const uint32_t xa = *reinterpret_cast<const uint16_t*>(own_scales + of * kMxBlocks);
            const Words4* ca = reinterpret_cast<const Words4*>(own + of * kMxBytes);
            acc = mma<0>(cb[i][0], xb[i], ca[0], xa, acc);
            acc = mma<1>(cb[i][1], xb[i], ca[1], xa, acc);
        }
    }
    finish_few<T>(sums, acc, out, 0, j0);
}

// Larger tiles: the operands in shared memory, two groups of k a step, in two stages
// that take turns.  First operand: b, whose rows are out's columns, so that a lane
// holds runs of a row of out.
constexpr int kMxStages = 2, kMxStep = 2;  // groups of a step

// kR rows of a group in shared memory.  The four 16-byte units of a row are permuted
// by the row where they come from, so that the eight lanes that read at once meet
// different banks.
template <class S, int kR>
struct MxStage {
    static constexpr int kLoads = kR * kMxBytes / 16 / S::kThreads;
    static constexpr int kBytes = kR * (kMxBytes + kMxBlocks);
    static_assert(kLoads * S::kThreads * 16 == kR * kMxBytes && kR <= S::kThreads && kR % 64 == 0, "whole loads");

    const Mx4& m;
    const char* codes;      // of the tile's first row
    const uint8_t* scales;
    uint32_t rows;          // from there on
    uint32_t unit;          // where this thread's first unit comes from

    __device__ __forceinline__ explicit MxStage(const Mx4& matrix) : m(matrix) {
        const uint32_t row = threadIdx.x / 4;
        unit = row * kMxBytes + ((threadIdx.x ^ row / 4) & 3) * 16;
    }
    __device__ __forceinline__ void place(int64_t first) {
        codes = m.codes + first * kMxBytes;
        scales = m.scales + first * kMxBlocks;
        rows = static_cast<uint32_t>(m.rows - first);
    }
    // Rows behind the last read as 0: their sums are not used.  So do all where there is
    // no such group (wanted false), without a read.
    __device__ __forceinline__ void load(int64_t g, bool wanted, MICRO_SHARED char* to) const {
        const uint32_t some = wanted ? rows : 0;
        const __amdgpu_buffer_rsrc_t from =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(codes + g * m.rows * kMxBytes), 0, some * kMxBytes, kRawBuffer);
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, to + (i * S::kThreads + wave * 64) * 16, 16,
                                                     unit + i * S::kThreads * 16, 0, 0, 0);
        const __amdgpu_buffer_rsrc_t words = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t*>(scales + g * m.rows * kMxBlocks), 0, some * kMxBlocks, kRawBuffer);
        // (a tile of fewer rows than threads: the same ones again)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(words, to + kR * kMxBytes + wave * 64 % kR * 4, 4,
                                                 threadIdx.x % kR * kMxBlocks, 0, 0, 0);
    }
    // Half h of a wavefront takes the blocks 2 h and 2 h + 1 of its rows.
    static __device__ __forceinline__ Words4 codes_at(MICRO_SHARED char* tile, int row, int kk) {
        const int half = threadIdx.x >> 5 & 1;
        return *(MICRO_SHARED Words4*)(tile + row * kMxBytes + ((half * 2 + kk) ^ (row / 4 & 3)) * 16);
    }
    static __device__ __forceinline__ uint32_t scales_at(MICRO_SHARED char* tile, int row) {
        return *(MICRO_SHARED uint16_t*)(tile + kR * kMxBytes + row * kMxBlocks + (threadIdx.x >> 5 & 1) * 2);
    }
};

template <class S>
struct MxTiles {
    using StageA = MxStage<S, S::kA>;
    using StageB = MxStage<S, S::kB>;
    // The tiles of a step's groups.
    struct Part {
        MICRO_SHARED char *a, *b;
    };
    struct Shared {
        Part stage[kMxStages][kMxStep];
    };
    struct Fragments {
        Words4 a[S::kTilesA], b[S::kTilesB];
    };
    struct Scales {
        uint32_t a[S::kTilesA], b[S::kTilesB];
        // Where there is no such group the least scales, 2^-254 together: whatever
        // codes they meet add less than half of binary32's least number.
        __device__ __forceinline__ void keep(bool there) {
            const uint32_t mask = there ? 0xffffffffu : 0;
#pragma unroll
            for (int i = 0; i < S::kTilesA; ++i) a[i] &= mask;
#pragma unroll
            for (int j = 0; j < S::kTilesB; ++j) b[j] &= mask;
        }
    };
    static constexpr int kReads = S::kTilesA + S::kTilesB, kProducts = S::kTilesA * S::kTilesB;
    static constexpr int kLoads = kMxStep * (StageA::kLoads + StageB::kLoads + 2);

    StageA sa;
    StageB sb;
    int64_t step, end;  // groups
    int row_a, row_b;   // the lane's first rows in the tiles

    __device__ __forceinline__ MxTiles(const Mx4& a, const Mx4& b) : sa(a), sb(b) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
        row_a = wave / S::kWavesB * (S::kTilesA * 32) + (lane & 31);
        row_b = wave % S::kWavesB * (S::kTilesB * 32) + (lane & 31);
    }

    __device__ __forceinline__ void load(int64_t g, const Part (&to)[kMxStep]) const {
#pragma unroll
        for (int i = 0; i < kMxStep; ++i) {
            sa.load(g + i, g + i < end, to[i].a);
            sb.load(g + i, g + i < end, to[i].b);
        }
    }
    // Until all but the last kPending of each wavefront's loads and stores are done (they
    // end in their order), where `more`, or else all; until what it has read from shared
    // memory is in registers; and until the others are here too.
    template <int kPending>
    static __device__ __forceinline__ void meet(bool more) {
        static_assert(kPending < 64, "the counter's bits");
        if (more)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kPending) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    static __device__ __forceinline__ void meet() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
    __device__ __forceinline__ void read(const Part& p, int kk, Fragments& f) const {
#pragma unroll
        for (int j = 0; j < S::kTilesB; ++j) f.b[j] = StageB::codes_at(p.b, row_b + j * 32, kk);
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i) f.a[i] = StageA::codes_at(p.a, row_a + i * 32, kk);
    }
    __device__ __forceinline__ void read(const Part& p, Scales& s) const {
#pragma unroll
        for (int j = 0; j < S::kTilesB; ++j) s.b[j] = StageB::scales_at(p.b, row_b + j * 32);
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i) s.a[i] = StageA::scales_at(p.a, row_a + i * 32);
    }
    template <int kk>
    static __device__ __forceinline__ void multiply(const Fragments& f, const Scales& s, Acc (&acc)[S::kTilesA][S::kTilesB]) {
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
            for (int j = 0; j < S::kTilesB; ++j) acc[i][j] = mma<kk>(f.a[i], s.a[i], f.b[j], s.b[j], acc[i][j]);
    }

    // The tile at (a, b), groups [first, until), of which the first step begins to
    // load.  All stages are free.
    __device__ __forceinline__ void start(int64_t a, int64_t b, int64_t first, int64_t until, const Shared& at) {
        step = first;
        end = until;
        sa.place(a);
        sb.place(b);
        load(step, at.stage[0]);
    }

    // acc += the sum.  Fragments are read while the matrix cores work on the ones
    // before.  stored: kStores stores at least lie behind start(); they need not be
    // done before the loads that follow them are waited for.
    template <int kStores>
    __device__ __forceinline__ void run(Acc (&acc)[S::kTilesA][S::kTilesB], const Shared& at, bool stored) {
        Fragments even, odd;
        Scales first, second;
        // All of a step but its last quarter.
        const auto work = [&](const Part (&p)[kMxStep]) {
            read(p[0], 1, odd);
            multiply<0>(even, first, acc);
            interleave<kProducts, kReads, 0>();
            read(p[1], second);
            read(p[1], 0, even);
            multiply<1>(odd, first, acc);
            interleave<kProducts, 2 * kReads, 0>();
            second.keep(step + 1 < end);
            read(p[1], 1, odd);
            multiply<0>(even, second, acc);
            interleave<kProducts, kReads, 0>();
        };
        // A step's last fragments are in registers before the barrier, so behind it
        // the loads of the step after next may overwrite its stage, and the next
        // step's first fragments are read, both under the step's last products.
        const auto turn = [&](const Part (&p)[kMxStep], const Part (&next)[kMxStep]) {
            meet();
            __builtin_amdgcn_sched_barrier(0);
            load(step + 2 * kMxStep, p);
            read(next[0], first);
            read(next[0], 0, even);
            multiply<1>(odd, second, acc);
            interleave<kProducts, 2 * kReads, kLoads>();
            step += kMxStep;
        };
        meet<kStores>(stored);
        load(step + kMxStep, at.stage[1]);
        read(at.stage[0][0], first);
        read(at.stage[0][0], 0, even);
        __builtin_amdgcn_sched_barrier(0);
        int64_t left = (end - step + 1) / kMxStep;
        for (; left > 2; left -= 2) {
            work(at.stage[0]);
            turn(at.stage[0], at.stage[1]);
            work(at.stage[1]);
            turn(at.stage[1], at.stage[0]);
        }
        work(at.stage[0]);
        if (left == 2) {
            meet();
            read(at.stage[1][0], first);
            read(at.stage[1][0], 0, even);
            multiply<1>(odd, second, acc);
            step += kMxStep;
            work(at.stage[1]);
        }
        multiply<1>(odd, second, acc);
        meet();  // the stages are free
    }
};

// One 16-byte chunk of a row of out, its values in [j, columns).
template <class T>
__device__ __forceinline__ void store_chunk(T* row, int64_t j, int64_t columns, Chunk x) {
    constexpr int kVec = 16 / sizeof(T);
    const Pack<T, kVec> v = __builtin_bit_cast(Pack<T, kVec>, x);
    if (j + kVec <= columns) {
        *reinterpret_cast<Pack<T, kVec>*>(row + j) = v;
    } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (j + i < columns) row[j + i] = v.v[i];
    }
}

struct MxOut {
    void* at;
    int64_t stride, rows, columns;
    bool accumulate;
    float* parts;
    int64_t most_splits;
};

// The 16-byte stores of a wavefront's whole tile, its least (binary32 and sums added
// to out take more).
template <class S>
constexpr int kLeastStores = S::kTilesB * S::kTilesA / 2 * 4;

// A finished tile's columns of matrix tiles from the j0-th on into out.
template <class S, class T, int kColumns>
__device__ __forceinline__ void finish_tile(const MxOut& out, MICRO_SHARED char* area, const Place<S>& place, int64_t ta,
                                            int64_t tb, int j0, Acc (&acc)[S::kTilesA][kColumns]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < kColumns; ++j) {
        const int64_t row0 = tb * S::kB + place.wave_b + (j0 + j) * 32 + (lane >> 3);
        if (sizeof(T) == 4 || out.accumulate) {
#pragma unroll
            for (int i = 0; i < S::kTilesA; ++i) {
                Chunk in[4], to[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const Vec4<float> x = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    in[q] = __builtin_bit_cast(Chunk, x);
                }
                exchange(area, in, to);
                const int64_t column = ta * S::kA + place.wave_a + i * 32 + (lane & 7) * 4;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int64_t r = row0 + 8 * k;
                    if (r >= out.rows || column >= out.columns) continue;
                    T* row = static_cast<T*>(out.at) + r * out.stride;
                    const Vec4<float> v = __builtin_bit_cast(Vec4<float>, to[k]);
                    if (column + 4 <= out.columns) {
                        float x[4] = {v[0], v[1], v[2], v[3]};
                        if (out.accumulate) {
                            float old[4];
                            load_floats(row + column, old);
#pragma unroll
                            for (int m = 0; m < 4; ++m) x[m] += old[m];
                        }
                        store_floats(row + column, x);
                    } else {
#pragma unroll
                        for (int m = 0; m < 4; ++m)
                            if (column + m < out.columns)
                                row[column + m] =
                                    rounded<T>(out.accumulate ? v[m] + static_cast<float>(row[column + m]) : v[m]);
                    }
                }
            }
        } else if constexpr (sizeof(T) == 2) {
            constexpr int kRun = 2;  // matrix tiles whose 16-bit values fill 128 bytes of a row
#pragma unroll
            for (int i = 0; i < S::kTilesA; i += kRun) {
                Chunk in[4], to[4];
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    if (i + m / 2 >= S::kTilesA) {
                        in[m] = Chunk{0, 0, 0, 0};
                        continue;
                    }
                    Vec4<T> lo, hi;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        lo[r] = rounded<T>(acc[i + m / 2][j][m % 2 * 8 + r]);
                        hi[r] = rounded<T>(acc[i + m / 2][j][m % 2 * 8 + 4 + r]);
                    }
                    swap_halves(lo, hi);
                    in[m] = __builtin_bit_cast(Chunk, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
                exchange(area, in, to);
                const int64_t column = ta * S::kA + place.wave_a + i * 32 + (lane & 7) * 8;
                const bool in_tile = (lane & 7) * 8 < (S::kTilesA - i) * 32;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int64_t r = row0 + 8 * k;
                    if (r < out.rows && column < out.columns && in_tile)
                        store_chunk(static_cast<T*>(out.at) + r * out.stride, column, out.columns, to[k]);
                }
            }
        }
    }
}

// Workgroups of a compute unit: what its shared memory holds.
template <class S>
constexpr int kMxPerUnit = 160 * 1024 / (kMxStages * kMxStep * (S::kA + S::kB) * (kMxBytes + kMxBlocks));

// Bound by the matrix cores, which are busy 57 to 67% of the cycles of a long sum, at a
// clock that sinks to 1.8 GHz under them: 8192 x 8192 x 8192 in 236 to 240 us (4.6 to 4.7
// PFLOP/s), 16384 x 8192 x 2048 in 123 to 128 (middle tiles 149 to 157), 16384 x 2048 x
// 8192, busy 44%, in 152 to 160 (191 to 195): a tile's eight steps take 13 us and its stores
// 6.  One group a step through four stages, with twice the barriers: 16384 x 8192 x 2048 in
// 127 where two groups took 124 (in middle tiles 190 for 157), 16384 x 2048 x 8192 in 163
// for 152.
template <class S, class T>
__global__ __launch_bounds__(S::kThreads) void product_kernel(Mx4 a, Mx4 b, MxOut out) {
    using Tiles = MxTiles<S>;
    // (each stage a variable of its own: that is how the compiler knows that reads of
    // one need not wait for the loads into another)
#define MICRO_MX_PART(name)                                                         \
    __shared__ __attribute__((aligned(1024))) char name##_a[Tiles::StageA::kBytes]; \
    __shared__ __attribute__((aligned(1024))) char name##_b[Tiles::StageB::kBytes]; \
    const typename Tiles::Part name{(MICRO_SHARED char*)name##_a, (MICRO_SHARED char*)name##_b}
    MICRO_MX_PART(part0);
    MICRO_MX_PART(part1);
    MICRO_MX_PART(part2);
    MICRO_MX_PART(part3);
    const typename Tiles::Shared at{{{part0, part1}, {part2, part3}}};
    TileOrder order((a.rows + S::kA - 1) / S::kA, (b.rows + S::kB - 1) / S::kB, out.most_splits);
    Tiles product(a, b);
    const Place<S> place;
    // the exchange of finished tiles, in the stage that start() leaves
    constexpr int kHalf = S::kThreads / 128;
    static_assert(kHalf * kExchange <= Tiles::StageA::kBytes && kHalf * kExchange <= Tiles::StageB::kBytes, "the exchange fits");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    MICRO_SHARED char* const area = (wave < kHalf ? part2.a : part2.b) + wave % kHalf * kExchange;
    const auto start = [&](const Tile& t) {
        const int64_t steps = (a.groups + kMxStep - 1) / kMxStep, parts = t.part < 0 ? 1 : order.splits;
        const int64_t part = t.part < 0 ? 0 : t.part, until = steps * (part + 1) / parts * kMxStep;
        product.start(t.a * S::kA, t.b * S::kB, steps * part / parts * kMxStep, until < a.groups ? until : a.groups, at);
    };
    Tile tile, after;
    bool more = order.next(&tile), full = false;
    if (more) start(tile);
    for (; more; tile = after) {
        Acc acc[S::kTilesA][S::kTilesB];
        clear<S>(acc);
        product.template run<kLeastStores<S>>(acc, at, full);
        more = order.next(&after);
        if (more) start(after);
        if (tile.part >= 0) {
#pragma unroll
            for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
                for (int j = 0; j < S::kTilesB; ++j) store_part<S>(tile_at<S>(out.parts, tile.index), i, j, acc[i][j]);
            full = false;
        } else {
            finish_tile<S, T, S::kTilesB>(out, area, place, tile.a, tile.b, 0, acc);
            full = (tile.a + 1) * S::kA <= out.columns && (tile.b + 1) * S::kB <= out.rows;
        }
    }
}

// Adds the parts of tiles whose sums were cut, in their order, a workgroup a column
// of matrix tiles of one wavefront.
template <class S, class T>
__global__ __launch_bounds__(64) void join_kernel(int64_t tiles_a, int64_t tiles_b, MxOut out, int64_t grid) {
    __shared__ __attribute__((aligned(1024))) char shared[kExchange];
    const TileOrder order(tiles_a, tiles_b, out.most_splits, grid);
    constexpr int kWaves = S::kThreads / 64;
    const int64_t t = blockIdx.x / (kWaves * S::kTilesB);
    if (t >= order.tail) return;
    const int of = blockIdx.x % (kWaves * S::kTilesB) / S::kTilesB, j = blockIdx.x % S::kTilesB;
    int64_t ta, tb;
    order.place(order.full + t, &ta, &tb);
    const Place<S> place(of);
    if (tb * S::kB + place.wave_b + j * 32 >= out.rows) return;
    Acc acc[S::kTilesA][1];
#pragma unroll
    for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][0][r] = 0.0f;
    for (int64_t s = 0; s < order.splits; ++s)
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i)
            add_part<S>(tile_at<S>(out.parts, s * order.tail + t, of * 64 + threadIdx.x), i, j, acc[i][0]);
    finish_tile<S, T, 1>(out, (MICRO_SHARED char*)shared, place, ta, tb, j, acc);
}

constexpr int64_t kMostGroups = int64_t(1) << 20;
dim3 grid_of(int64_t n) { return dim3(static_cast<uint32_t>(std::min(n, kMostGroups))); }

dim3 grid_of(int64_t x, int64_t y) {
    return dim3(static_cast<uint32_t>(x), static_cast<uint32_t>(std::min<int64_t>(y, 65535)));
}

template <class T>
hipError_t pack(const Rows& x, const Mx4& packed, const Mx4& turned, hipStream_t stream) {
    const T* at = static_cast<const T*>(x.at);
    if (!turned.codes)
        return launch(pack_kernel<T>,
                      grid_of((packed.groups + kPackGroups - 1) / kPackGroups, (packed.rows + kPackRows - 1) / kPackRows),
                      kPackThreads, stream, at, x.stride, packed);
    return launch(packed.codes ? pack_turned_kernel<T, true> : pack_turned_kernel<T, false>,
                  grid_of((turned.rows + kTurnColumns - 1) / kTurnColumns, turned.groups), kPackThreads, stream, at, x.stride,
                  packed, turned);
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
    const dim3 grid = grid_of((from.rows * from.groups + kPackThreads / kPackLanes - 1) / (kPackThreads / kPackLanes));
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

constexpr int64_t kPartGroups = 32;

// The product in tiles of shape S by a grid that fills the card.
template <class S, class T>
hipError_t tiles(const Mx4Product& c, hipStream_t stream) {
    const int64_t ta = (c.b.rows + S::kA - 1) / S::kA, tb = (c.a.rows + S::kB - 1) / S::kB;
    const int64_t grid = c.compute_units / TileOrder::kDies * TileOrder::kDies * kMxPerUnit<S>;
    static_assert(S::kA * S::kB * kMxPerUnit<S> <= kMxParts, "the parts of a grid fit");
    MxOut out{c.out.at, c.out.stride, c.a.rows, c.b.rows, c.accumulate, c.parts, 1};
    // The tiles behind the last full round are cut along the sum where they are a quarter
    // of the grid at most and a part keeps kPartGroups: writing and adding the parts costs
    // more than it saves else (1024 x 16384 x 1024 in 23.6 us for 41.5, but 1024 x 8192 x
    // 4096 in 34.2 for 26.7).
    const int64_t tail = ta * tb % grid;
    if (tail > 0 && tail * 4 <= grid) out.most_splits = std::min(grid / tail, std::max<int64_t>(c.a.groups / kPartGroups, 1));
    if (const hipError_t e = launch(product_kernel<S, T>, dim3(static_cast<uint32_t>(grid)), S::kThreads, stream, c.b, c.a, out))
        return e;
    if (out.most_splits <= 1) return hipSuccess;
    return launch(join_kernel<S, T>, dim3(static_cast<uint32_t>(tail * (S::kThreads / 64) * S::kTilesB)), 64, stream, ta, tb,
                  out, grid);
}

// How long `tiles` tiles take: rounds of a full grid, and the less that the last one
// takes when it is not full, in microseconds for each step of long sums (16384 x 16384 x
// 4096: 8 rounds of middle tiles in 565 us, 4 of wide ones in 459; one round that is not
// full 0.6 to 0.7 and 1.2).  Where the stores weigh as much as the sums the same side is
// the faster one at what was measured: 4096 x 2048 x 50257 in wide tiles 313 us, in middle
// ones 338, 16384 x 2048 x 8192 153 and 191, 1000 x 1024 x 4096 12.6 and 8.8, 1024 x 256 x
// 4096 9.3 and 7.2.
double rounds(int64_t tiles, int64_t grid, double full, double rest) {
    return tiles / grid * full + (tiles % grid ? rest : 0.0);
}

// Tiles of 32 x 32 that are better off one a workgroup, whose wavefronts share the sum,
// while they and their groups are few: 256 x 2048 x 1024 takes 4.6 us for 9.4 in middle
// tiles, 256 x 8192 x 1024 9.7 for 16.5, 256 x 2048 x 4096 9.7 both, 512 x 2048 x 4096 14.7
// for 10.2, 1024 x 256 x 4096 10.8 for 7.2.  The border is not that of every shape: 256 x
// 16384 x 1024, behind it, takes 18.3 in middle tiles and would take 15.1.
//   Rows that the workgroups pack themselves save a launch: twice as many groups.  Calls
// from x, of tables that come from memory, in us by rows of their own / by a packing launch
// and middle tiles:
//   1 x 2048 x 30522    7.8 / 14.1      1 x 4096 x 50257   23.3 / 28.3
//   1 x 2048 x 50257   13.3 / 18.4      1 x 2048 x 131072  31.9 / 34.2
//   1 x 2048 x 65536   16.6 / 19.0      1 x 1024 x 262144  32.2 / 39.0
//   4 x 2048 x 65536   19.5 / 19.7      1 x 4096 x 131072  60.7 / 57.3 (5.0 TB/s)
// and of up to 32 rows that a launch packs, in tiles of 32 x 32 / middle ones:
//   19 x 2048 x 30522  12.8 / 15.0      19 x 4096 x 50257  30.8 / 27.5
//   19 x 2048 x 50257  19.3 / 19.2      19 x 2048 x 131072 40.5 / 35.1
//   32 x 2048 x 50257  21.2 / 19.7      19 x 4096 x 131072 75.5 / 60.5
// Behind the limits (the right column; 19 and 32 x 2048 x 50257) middle tiles are what
// runs: one to four rows lose up to a fifth by it, more rows gain.
constexpr int64_t kFewTiles = 2048, kFewGroups = 16384, kOwnGroups = 2 * kFewGroups;

int64_t few_tiles(const Mx4Product& c) {
    return (c.a.rows + kTile - 1) / kTile * ((c.b.rows + kTile - 1) / kTile);
}
bool takes_few(const Mx4Product& c, int64_t most_groups = kFewGroups) {
    const int64_t few = few_tiles(c);
    return (few <= kFewTiles && few * c.a.groups <= most_groups) || c.a.groups == 0;
}
FewOut few_out(const Mx4Product& c) { return {c.out.at, c.out.stride, c.a.rows, c.b.rows, c.accumulate}; }

template <class X>
hipError_t few_linear(const X* x, int64_t stride, const Mx4Product& c, hipStream_t stream) {
    const auto kernel = c.out.type == MICRO_TYPE_F32   ? few_linear_kernel<X, float>
                        : c.out.type == MICRO_TYPE_F16 ? few_linear_kernel<X, f16>
                                                       : few_linear_kernel<X, bf16>;
    return launch(kernel, grid_of(few_tiles(c)), 64 * kFewWaves, stream, x, stride, static_cast<int>(c.a.rows), c.b, few_out(c));
}

template <class T>
hipError_t product(const Mx4Product& c, hipStream_t stream) {
    if (takes_few(c))
        return launch(few_kernel<T>, grid_of(few_tiles(c)), 64 * kFewWaves, stream, c.a, c.b, few_out(c));
    const auto count = [&](int64_t a, int64_t b) { return (c.b.rows + a - 1) / a * ((c.a.rows + b - 1) / b); };
    const double middle = rounds(count(Middle::kA, Middle::kB), c.compute_units * kMxPerUnit<Middle>, 1.1, 0.7);
    const double wide = rounds(count(Wide::kA, Wide::kB), c.compute_units * kMxPerUnit<Wide>, 1.77, 1.25);
    return wide < middle ? tiles<Wide, T>(c, stream) : tiles<Middle, T>(c, stream);
}

}  // namespace

hipError_t launch_mx4_linear(const Rows& x, const Mx4Product& c, hipStream_t stream) {
    if (c.a.rows > 0 && c.a.rows <= kTile && c.b.rows > 0 && c.a.groups > 0 && c.a.rows * c.a.groups * kMxGroup <= kOwnValues &&
        takes_few(c, kOwnGroups)) {
        switch (x.type) {
            case MICRO_TYPE_F32: return few_linear(static_cast<const float*>(x.at), x.stride, c, stream);
            case MICRO_TYPE_F16: return few_linear(static_cast<const f16*>(x.at), x.stride, c, stream);
            default: return few_linear(static_cast<const bf16*>(x.at), x.stride, c, stream);
        }
    }
    if (const hipError_t e = launch_mx4_pack(x, c.a.rows, c.a.cols, c.a, Mx4{}, stream)) return e;
    return launch_mx4_product(c, stream);
}

hipError_t launch_mx4_product(const Mx4Product& c, hipStream_t stream) {
    if (c.a.rows == 0 || c.b.rows == 0) return hipSuccess;
    switch (c.out.type) {
        case MICRO_TYPE_F32: return product<float>(c, stream);
        case MICRO_TYPE_F16: return product<f16>(c, stream);
        default: return product<bf16>(c, stream);
    }
}

}  // namespace micro

// Device-side tiles of matrix products on gfx950's matrix cores, for the kernels of
// the token loss and of the 4-bit products: operand tiles in shared memory, the
// order in which a grid takes tiles, and how finished ones leave.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "value_types.h"

namespace micro {

// A row of an operand's tile is this many 16-bit values, 128 bytes.
constexpr int kDepth = 64;

template <class T>
using Vec8 = T __attribute__((ext_vector_type(8)));
template <class T>
using Vec4 = T __attribute__((ext_vector_type(4)));
using Acc = float __attribute__((ext_vector_type(16)));

#define MICRO_SHARED __attribute__((address_space(3)))
// The last word of a raw buffer's descriptor: untyped, 32-bit elements.
constexpr int kRawBuffer = 0x00027000;

template <class T>
__device__ __forceinline__ Vec4<T> read_transposed(MICRO_SHARED char* p) {
    return __builtin_bit_cast(Vec4<T>, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MICRO_SHARED Vec4<short>*)p));
}

// One operand.  Straight: rows of the kept axis, k adjacent.  Turned: rows of
// k, the kept axis adjacent.
struct Operand {
    const void* at;
    int64_t stride;  // values between rows
    int64_t kept;    // valid values of the kept axis (turned: a multiple of 8)
    int64_t depth;   // turned: valid rows of k; those behind read the last one
    int64_t plane;   // values between the planes of a split operand
};

// A workgroup of kWavesA x kWavesB wavefronts, each with kTilesA x kTilesB
// matrix tiles of 32 x 32.
template <int WA, int WB, int TA, int TB>
struct Shape {
    static constexpr int kWavesA = WA, kWavesB = WB, kTilesA = TA, kTilesB = TB;
    static constexpr int kThreads = 64 * WA * WB;
    static constexpr int kA = WA * TA * 32, kB = WB * TB * 32;  // the tile of C
    static_assert(kA * kDepth * 2 >= WA * WB * 4096, "the exchange fits a tile of a");
    static constexpr int kPerUnit = 160 * 1024 / (2 * (kA + kB) * kDepth * 2);  // workgroups of a compute unit
};
using Wide = Shape<2, 4, 4, 2>;
using Middle = Shape<2, 2, 2, 2>;
using Narrow32 = Shape<4, 1, 1, 1>;

// The tile of an operand in shared memory: kR values of the kept axis by
// kDepth of k, filled by loads that go from global to shared memory without
// registers, 16 bytes a lane and the lanes of a wavefront in order.  So that
// fragments are read without bank conflicts the 16-byte units of a row are
// permuted where they come from: straight rows by the row, turned rows (in
// pairs of units) by k.
template <class T, int kR, bool kTurned, int kThreads>
struct Stage {
    static constexpr int kLoads = kR * kDepth / 8 / kThreads;
    static_assert(kLoads * kThreads * 8 == kR * kDepth, "a tile is a whole number of loads");
    static constexpr int kRowUnits = kTurned ? kR / 8 : kDepth / 8;
    static constexpr uint32_t kRowsPerLoad = kThreads / kRowUnits;
    // a thread's unit has the same place in each of its rows
    static_assert(kThreads % kRowUnits == 0 && kRowsPerLoad % 16 == 0, "rows of a load");

    // The four rows of k that a group of lanes reads together lie 2 kR bytes
    // apart; what to permute a turned row's pairs by so that they do not meet
    // in the same 256 bytes of banks.
    static constexpr __device__ uint32_t swizzle(uint32_t k) { return kR >= 128 ? (k & 3) * 2 : kR == 64 ? (k & 2) : 0; }

    uint32_t row, unit;     // this thread's first row, and the bytes of its unit in a row
    uint32_t stride, last;  // bytes between rows; straight: the last valid row

    __device__ void place(const Operand& op, int64_t first) {
        const uint32_t kept = static_cast<uint32_t>(op.kept - first < kR ? op.kept - first : kR);
        row = threadIdx.x / kRowUnits;
        uint32_t u = threadIdx.x % kRowUnits;
        if constexpr (kTurned) {
            u ^= swizzle(row) * 2;
            u = u * 8 + 8 <= kept ? u : kept / 8 - 1;
        } else {
            u ^= (row >> 1) & 7;
        }
        unit = u * 16;
        stride = static_cast<uint32_t>(op.stride * sizeof(T));
        last = kept - 1;
    }

    // last_row: of this step.  Rows behind it are read from it: what they are
    // multiplied with is zero (k), or the result is not used (the kept axis).
    // Both factors have at most 24 bits.
    __device__ __forceinline__ void load(const char* from, MICRO_SHARED char* to, uint32_t last_row) const {
        const __amdgpu_buffer_rsrc_t rows =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from), 0, -1, kRawBuffer);
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t r = row + i * kRowsPerLoad;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, to + (i * kThreads + wave * 64) * 16, 16,
                                                     __umul24(r < last_row ? r : last_row, stride) + unit, 0, 0, 0);
        }
    }

    // Values [base, base + 32) of the kept axis by k [kk * 16, + 16): lane l
    // holds value l % 32 and the eight k from 8 * (l / 32).
    static __device__ __forceinline__ Vec8<T> fragment(MICRO_SHARED char* tile, int base, int kk) {
        const int lane = threadIdx.x & 63;
        if constexpr (kTurned) {
            // four k by 16 values transposed by each group of 16 lanes, twice
            const int k = kk * 16 + (lane >> 5) * 8 + ((lane & 15) >> 2);
            const int pair = (base >> 4) + ((lane >> 4) & 1);
            const int at = (k * kR + (pair ^ swizzle(k)) * 16 + (lane & 3) * 4) * int(sizeof(T));
            const Vec4<T> lo = read_transposed<T>(tile + at), hi = read_transposed<T>(tile + (at + 4 * kR * int(sizeof(T))));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            const int r = base + (lane & 31), c = kk * 2 + (lane >> 5);
            return *(MICRO_SHARED Vec8<T>*)unit_at(tile, r, c);
        }
    }

    // The 16-byte unit c of a straight row.
    static __device__ __forceinline__ MICRO_SHARED char* unit_at(MICRO_SHARED char* tile, int r, int c) {
        return tile + (r * (kDepth * 2) + (c ^ ((r >> 1) & 7)) * 16);
    }
};

// Orders the instructions since the last such call: reads of shared memory and
// loads spread between the products, whose 32 cycles each cover their issue.
template <int kProducts, int kReads, int kLoads, int kAt = 0>
__device__ __forceinline__ void interleave() {
    if constexpr (kAt < kProducts) {
        constexpr int kMma = 0x8, kVectorLoad = 0x20, kSharedRead = 0x100;
        __builtin_amdgcn_sched_group_barrier(kMma, 1, 0);
        // the reads in the first half, so that the next products do not wait for them
        constexpr int kHalf = kProducts < 8 ? kProducts : 4, each = (kReads + kHalf - 1) / kHalf;
        constexpr int reads = kAt * each >= kReads ? 0 : kReads - kAt * each < each ? kReads - kAt * each : each;
        constexpr int loads = (kAt + 1) * kLoads / kProducts - kAt * kLoads / kProducts;
        if constexpr (loads > 0) __builtin_amdgcn_sched_group_barrier(kVectorLoad, loads, 0);
        if constexpr (reads > 0) __builtin_amdgcn_sched_group_barrier(kSharedRead, reads, 0);
        interleave<kProducts, kReads, kLoads, kAt + 1>();
    } else {
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The two operands' tiles of a stage.  While a tile of C is finished, the first
// stage is already being filled for the next and the second one's tile of a
// serves the exchange.  Each tile of each stage is a variable of
// its own: that is how the compiler knows that reads of one stage need not wait
// for the loads into the other.
struct Tiles {
    MICRO_SHARED char *a, *b;
};
#define MICRO_STAGES(S)                                                        \
    __shared__ __attribute__((aligned(1024))) char tile_a0[S::kA * kDepth * 2]; \
    __shared__ __attribute__((aligned(1024))) char tile_b0[S::kB * kDepth * 2]; \
    __shared__ __attribute__((aligned(1024))) char tile_a1[S::kA * kDepth * 2]; \
    __shared__ __attribute__((aligned(1024))) char tile_b1[S::kB * kDepth * 2]; \
    const Tiles stage0{(MICRO_SHARED char*)tile_a0, (MICRO_SHARED char*)tile_b0}; \
    const Tiles stage1{(MICRO_SHARED char*)tile_a1, (MICRO_SHARED char*)tile_b1}

template <class S>
__device__ void clear(Acc (&acc)[S::kTilesA][S::kTilesB]) {
#pragma unroll
    for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
        for (int j = 0; j < S::kTilesB; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
}

// Where a lane's four adjacent values acc[i][j][4 q .. 4 q + 3] lie in C.
template <class S>
struct Place {
    int wave_a, wave_b;  // the wavefront's first value in the tile
    int a, b;            // the lane's
    __device__ explicit Place(int wave = threadIdx.x >> 6) {
        const int lane = threadIdx.x & 63;
        wave_a = wave / S::kWavesB * (S::kTilesA * 32);
        wave_b = wave % S::kWavesB * (S::kTilesB * 32);
        a = wave_a + (lane >> 5) * 4;
        b = wave_b + (lane & 31);
    }
    __device__ int row(int i, int q) const { return a + i * 32 + q * 8; }
    __device__ int column(int j) const { return b + j * 32; }
};

// Eight values of a lane, 4 of one run of 8 and 4 of the next, become 8
// adjacent ones: the lower half of the wavefront ends up with the first run,
// the upper with the second.
template <class V>
__device__ __forceinline__ void swap_halves(V& first, V& second) {
    constexpr int kWords = sizeof(V) / 4;
    using Words = uint32_t __attribute__((ext_vector_type(kWords)));
    Words x = __builtin_bit_cast(Words, first), y = __builtin_bit_cast(Words, second);
#pragma unroll
    for (int w = 0; w < kWords; ++w) {
        const auto both = __builtin_amdgcn_permlane32_swap(x[w], y[w], false, false);
        x[w] = both[0];
        y[w] = both[1];
    }
    first = __builtin_bit_cast(V, x);
    second = __builtin_bit_cast(V, y);
}

using Chunk = uint32_t __attribute__((ext_vector_type(4)));  // 16 bytes
constexpr int kExchange = 4096;                               // shared memory of a wavefront's exchange

// 32 rows of C by 128 bytes change hands within a wavefront.  In: lane l holds
// of row l % 32 the chunks 2 m + l / 32.  Out: chunk l % 8 of the rows 8 k + l /
// 8, so that a store covers whole 128-byte lines of eight rows.  The chunks are
// permuted like a straight tile's.  `area` is the wavefront's own.
__device__ __forceinline__ void exchange(MICRO_SHARED char* area, const Chunk (&in)[4], Chunk (&out)[4]) {
    const int lane = threadIdx.x & 63;
    const int row = lane & 31, upper = lane >> 5;
#pragma unroll
    for (int m = 0; m < 4; ++m)
        *(MICRO_SHARED Chunk*)(area + row * 128 + ((2 * m + upper) ^ ((row >> 1) & 7)) * 16) = in[m];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = 8 * k + (lane >> 3);
        out[k] = *(MICRO_SHARED Chunk*)(area + r * 128 + ((lane & 7) ^ ((r >> 1) & 7)) * 16);
    }
    __builtin_amdgcn_wave_barrier();
}

// The tiles of C for a grid of workgroups that each take several, in rounds of
// one tile a workgroup.  The tiles behind the last full round are cut into
// `splits` parts of the summed axis, so that they too keep the grid busy.
// Workgroups go to the eight dies in turn, and each die has its own L2: a die
// takes a run of neighbouring tiles, ordered so that those in flight at once
// (four along a by the rest along b) share their operands.
struct Tile {
    int64_t a, b;
    int64_t part;   // of its sum; -1: the whole tile
    int64_t index;  // of the part among all parts
};
struct TileOrder {
    static constexpr int kDies = 8, kGroup = 4;
    int64_t tiles_a, tiles_b, full, tail, splits, round = 0;
    __device__ TileOrder(int64_t ta, int64_t tb, int64_t most_splits, int64_t grid = gridDim.x) : tiles_a(ta), tiles_b(tb) {
        const int64_t tiles = ta * tb;
        full = tiles / grid * grid;
        tail = tiles - full;
        splits = 1;
        if (tail > 0 && most_splits > 1) splits = grid / tail < most_splits ? grid / tail : most_splits;
    }
    __device__ void place(int64_t linear, int64_t* a, int64_t* b) const {
        const int64_t group = linear / (kGroup * tiles_b), rest = linear - group * (kGroup * tiles_b);
        const int64_t width = tiles_a - group * kGroup < kGroup ? tiles_a - group * kGroup : kGroup;
        *b = rest / width;
        *a = group * kGroup + (rest - *b * width);
    }
    __device__ bool next(Tile* t) {
        const int64_t grid = gridDim.x, die = blockIdx.x % kDies, in_die = blockIdx.x / kDies;
        if (round * grid < full) {
            place(die * (full / kDies) + in_die + round * (grid / kDies), &t->a, &t->b);
            t->part = -1;
            ++round;
            return true;
        }
        if (round * grid > full) return false;
        ++round;
        const int64_t parts = tail * splits, per_die = (parts + kDies - 1) / kDies;
        const int64_t at = die * per_die + in_die;
        if (in_die >= per_die || at >= parts) return false;
        place(full + at % tail, &t->a, &t->b);
        t->part = splits > 1 ? at / tail : -1;
        t->index = at;
        return true;
    }
};

template <class S>
__device__ float4* tile_at(float* tiles, int64_t index, int thread = threadIdx.x) {
    return reinterpret_cast<float4*>(tiles + index * (S::kA * S::kB)) + thread;
}

// The part (i, j) of a tile held as one float4 a thread and four rows.
template <class S>
__device__ __forceinline__ void store_part(float4* to, int i, int j, const Acc& acc) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
        to[((i * S::kTilesB + j) * 4 + q) * S::kThreads] =
            make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
}

template <class S>
__device__ __forceinline__ void add_part(const float4* from, int i, int j, Acc& acc) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float4 x = from[((i * S::kTilesB + j) * 4 + q) * S::kThreads];
        acc[4 * q] += x.x;
        acc[4 * q + 1] += x.y;
        acc[4 * q + 2] += x.z;
        acc[4 * q + 3] += x.w;
    }
}

}  // namespace micro

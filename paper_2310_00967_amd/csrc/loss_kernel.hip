// gfx950 kernels of the softmax cross entropy over a token table and of its
// gradients:
//   l_tv = h_t . W_v,   lse_t = log sum_v exp l_tv,   loss_t = lse_t - l_ty
//   g_tv = exp(l_tv - lse_t) - [v = y_t]
//   dh = f g W,   dW = f g^T h,   f = scale, or scale / counted tokens
// Three products of tokens, vocabulary and width on the matrix cores, in
// blocks of tokens: a block's exponentials exist as 16-bit codes, the logits
// themselves never leave the registers.  Each granule of vocabulary rows is
// normalised by its own maximum, and the granules are joined per token
// afterwards, so one pass over the table gives both the loss and what the
// gradients need.  Tokens that do not count are left out before the first
// product: everything below runs over the counted tokens only, whose number
// stays on the device.
//
// binary32 operands are split into three bfloat16 terms (24 bits of
// significand); a product is the sum of the six products of terms whose
// weights are above 2^-24, accumulated in binary32 like the others.
#include "loss_kernel.h"

#include <algorithm>

#include "launch.h"
#include "micro_sparsify.h"
#include "value_types.h"

namespace micro {
namespace {

constexpr int kDepth = kProductDepth;
constexpr float kLog2e = 1.44269504088896340736f;

template <class T>
using Vec8 = T __attribute__((ext_vector_type(8)));
template <class T>
using Vec4 = T __attribute__((ext_vector_type(4)));
using Acc = float __attribute__((ext_vector_type(16)));

#define MICRO_SHARED __attribute__((address_space(3)))
// The last word of a raw buffer's descriptor: untyped, 32-bit elements.
constexpr int kRawBuffer = 0x00027000;

__device__ __forceinline__ Acc mma(Vec8<bf16> a, Vec8<bf16> b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ Acc mma(Vec8<f16> a, Vec8<f16> b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
template <class T>
__device__ __forceinline__ Vec4<T> read_transposed(MICRO_SHARED char* p) {
    return __builtin_bit_cast(Vec4<T>, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MICRO_SHARED Vec4<short>*)p));
}

// ---------------------------------------------------------------------------
// the product C[a][b] = sum_k A[a][k] B[b][k]
// ---------------------------------------------------------------------------

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
            return *(MICRO_SHARED Vec8<T>*)(tile + (r * (kDepth * 2) + (c ^ ((r >> 1) & 7)) * 16));
        }
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

// The planes of a and b of a split operand's six products, four bits each;
// the first is that of a plain one.
constexpr uint32_t kPlanesA = 0x201100, kPlanesB = 0x021010;

// The product of one tile of C after another.  start() begins the loads of a
// tile's first step; run() is its sum.  In between a workgroup finishes the
// tile before, from registers.
template <class S, class T, int kTerms, bool kTurnA, bool kTurnB>
struct Product {
    using StageA = Stage<T, S::kA, kTurnA, S::kThreads>;
    using StageB = Stage<T, S::kB, kTurnB, S::kThreads>;
    // The fragments of 16 k, read while the matrix cores work on the 16 before.
    struct Fragments {
        Vec8<T> a[S::kTilesA], b[S::kTilesB];
    };
    static constexpr int kReads = (kTurnA ? 2 : 1) * S::kTilesA + (kTurnB ? 2 : 1) * S::kTilesB;
    static constexpr int kProducts = S::kTilesA * S::kTilesB, kLoads = StageA::kLoads + StageB::kLoads;
    static_assert(kDepth == 64, "four fragments a step");

    const Operand& A;
    const Operand& B;
    const int64_t blocks;
    StageA sa;
    StageB sb;
    const char *at_a, *at_b;
    int64_t step, end;

    __device__ __forceinline__ Product(const Operand& a, const Operand& b, int64_t blocks_of_k)
        : A(a), B(b), blocks(blocks_of_k) {}

    static __device__ __forceinline__ uint32_t last_row(int64_t depth, int64_t k) {
        const int64_t left = depth - k * kDepth;
        return static_cast<uint32_t>(left < kDepth ? left : kDepth) - 1;
    }
    // Step s is block s % blocks of k of term pair s / blocks.
    __device__ __forceinline__ void load(int64_t s, const Tiles& stage) const {
        const int term = kTerms == 1 ? 0 : static_cast<int>(s / blocks);
        const int64_t k = s - term * blocks;
        const int64_t step_a = (kTurnA ? A.stride * kDepth : kDepth), step_b = (kTurnB ? B.stride * kDepth : kDepth);
        sa.load(at_a + ((kPlanesA >> 4 * term & 15) * A.plane + k * step_a) * int64_t(sizeof(T)), stage.a,
                kTurnA ? last_row(A.depth, k) : sa.last);
        sb.load(at_b + ((kPlanesB >> 4 * term & 15) * B.plane + k * step_b) * int64_t(sizeof(T)), stage.b,
                kTurnB ? last_row(B.depth, k) : sb.last);
    }
    static __device__ __forceinline__ void arrived() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
    static __device__ __forceinline__ void read(const Tiles& stage, int kk, Fragments& f) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int a = wave / S::kWavesB * (S::kTilesA * 32), b = wave % S::kWavesB * (S::kTilesB * 32);
#pragma unroll
        for (int j = 0; j < S::kTilesB; ++j) f.b[j] = StageB::fragment(stage.b, b + j * 32, kk);
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i) f.a[i] = StageA::fragment(stage.a, a + i * 32, kk);
    }
    static __device__ __forceinline__ void multiply(const Fragments& f, Acc (&acc)[S::kTilesA][S::kTilesB]) {
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
            for (int j = 0; j < S::kTilesB; ++j) acc[i][j] = mma(f.a[i], f.b[j], acc[i][j]);
    }

    // The tile at (a, b), steps [first, until).  The stages are free.
    __device__ __forceinline__ void start(int64_t a, int64_t b, int64_t first, int64_t until, const Tiles& stage0) {
        step = first;
        end = until;
        if (step >= end) return;
        sa.place(A, a);
        sb.place(B, b);
        at_a = static_cast<const char*>(A.at) + (kTurnA ? a : a * A.stride) * int64_t(sizeof(T));
        at_b = static_cast<const char*>(B.at) + (kTurnB ? b : b * B.stride) * int64_t(sizeof(T));
        load(step, stage0);
    }

    // acc += the sum.  Two stages of shared memory: while the matrix cores work
    // on one, the loads of the next step fill the other.
    __device__ __forceinline__ void run(Acc (&acc)[S::kTilesA][S::kTilesB], const Tiles& stage0, const Tiles& stage1) {
        if (step >= end) return;
        Fragments even, odd;
        // All of a step but its last product.
        const auto work = [&](const Tiles& stage) {
            read(stage, 1, odd);
            multiply(even, acc);
            interleave<kProducts, kReads, 0>();
            read(stage, 2, even);
            multiply(odd, acc);
            interleave<kProducts, kReads, 0>();
            read(stage, 3, odd);
            multiply(even, acc);
            interleave<kProducts, kReads, 0>();
        };
        // A step's last fragments are in registers before the barrier, so behind
        // it the loads of the step after next may overwrite its stage, and the
        // next step's first fragments are read, both under the step's last
        // product.
        const auto turn = [&](int64_t to_load, const Tiles& stage, const Tiles& next) {
            arrived();
            __builtin_amdgcn_sched_barrier(0);
            load(to_load, stage);
            read(next, 0, even);
            multiply(odd, acc);
            interleave<kProducts, kReads, kLoads>();
        };
        int64_t left = end - step;
        const int64_t last = end - 1;
        arrived();
        load(step + 1 < last ? step + 1 : last, stage1);
        read(stage0, 0, even);
        __builtin_amdgcn_sched_barrier(0);
        for (; left > 2; left -= 2, step += 2) {
            work(stage0);
            turn(step + 2, stage0, stage1);
            work(stage1);
            turn(step + 3 < last ? step + 3 : last, stage1, stage0);  // past the end: the last step again
        }
        work(stage0);
        if (left == 2) {
            arrived();
            read(stage1, 0, even);
            multiply(odd, acc);
            work(stage1);
        }
        multiply(odd, acc);
        arrived();  // the stages are free
    }
};

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

// ---------------------------------------------------------------------------
// before the products
// ---------------------------------------------------------------------------

__device__ __forceinline__ int64_t target_of(const TokenIds& ids, int64_t t) {
    return ids.wide ? static_cast<const int64_t*>(ids.at)[t] : static_cast<const int32_t*>(ids.at)[t];
}

// Tokens of a chunk, whose counted ones are counted together.
constexpr int kChunkTokens = 1024;
// A target outside the vocabulary in a chunk, beside its count.
constexpr uint32_t kOutside = 0x80000000u;

struct Targets {
    TokenIds ids;
    int64_t tokens, ignored, vocab;
    __device__ bool counts(int64_t y) const { return y != ignored && y >= 0 && y < vocab; }
    __device__ bool outside(int64_t y) const { return y != ignored && (y < 0 || y >= vocab); }
};

__global__ __launch_bounds__(kChunkTokens) void count_kernel(Targets targets, uint32_t* chunks) {
    __shared__ int32_t waves[kChunkTokens / 64];
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kChunkTokens + threadIdx.x;
    const int64_t y = t < targets.tokens ? target_of(targets.ids, t) : targets.ignored;
    const uint64_t all = __ballot(targets.counts(y));
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = __popcll(all);
    const int any = __syncthreads_or(targets.outside(y));
    if (threadIdx.x != 0) return;
    uint32_t sum = 0;
    for (int w = 0; w < kChunkTokens / 64; ++w) sum += waves[w];
    chunks[blockIdx.x] = sum | (any ? kOutside : 0);
}

// x as a + b + c.  A first term that would round past bfloat16's range is cut
// instead.  An infinity or a NaN goes into the last term, which meets only the
// other operand's first: its product is what x's own would be, and no term of
// zero meets it.
__device__ __forceinline__ void split3(float x, bf16& a, bf16& b, bf16& c) {
    const uint32_t bits = __float_as_uint(x);
    a = static_cast<bf16>(x);
    if (!__builtin_isfinite(static_cast<float>(a))) a = __builtin_bit_cast(bf16, static_cast<uint16_t>(bits >> 16));
    const float r = x - static_cast<float>(a);
    b = static_cast<bf16>(r);
    c = static_cast<bf16>(r - static_cast<float>(b));
    if ((bits & 0x7f800000u) == 0x7f800000u) {
        c = static_cast<bf16>(x);
        a = b = static_cast<bf16>(0.0f);
    }
}

// One row of `dim` values into `padded` values of each plane, zeros behind, by
// `threads` threads.
template <class T>
__device__ void copy_row(const T* from, int dim, T* to, int padded, int64_t, int thread, int threads) {
    constexpr int kAhead = 4;
    int c = thread * 8;
    for (; c + (kAhead - 1) * threads * 8 + 8 <= dim; c += kAhead * threads * 8) {
        Pack<T, 8> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) x[u] = *reinterpret_cast<const Pack<T, 8>*>(from + c + u * threads * 8);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) *reinterpret_cast<Pack<T, 8>*>(to + c + u * threads * 8) = x[u];
    }
    for (; c < padded; c += threads * 8) {
        Pack<T, 8> x;
        if (c + 8 <= dim)
            x = *reinterpret_cast<const Pack<T, 8>*>(from + c);
        else
            for (int j = 0; j < 8; ++j) x.v[j] = c + j < dim ? from[c + j] : static_cast<T>(0.0f);
        *reinterpret_cast<Pack<T, 8>*>(to + c) = x;
    }
}
__device__ inline void copy_row(const float* from, int dim, bf16* to, int padded, int64_t plane, int thread, int threads) {
    for (int c = thread * 4; c < padded; c += threads * 4) {
        Pack<bf16, 4> p[kSplitPlanes];
        for (int j = 0; j < 4; ++j)
            split3(c + j < dim ? from[c + j] : 0.0f, p[0].v[j], p[1].v[j], p[2].v[j]);
        for (int q = 0; q < kSplitPlanes; ++q) *reinterpret_cast<Pack<bf16, 4>*>(to + q * plane + c) = p[q];
    }
}

constexpr int kRowBlock = 256, kGathered = kRowBlock / 64;  // a token a wavefront

struct Selection {
    const uint32_t* chunks;  // of count_kernel; not read for the tokens of one chunk
    int32_t* count;          // out: counted tokens; whether a target lies outside; 0 (softmax_kernel's arrivals)
    int32_t* rows;           // out
    int32_t* labels;         // out
    float* losses;           // out: 0 for an ignored token, NaN for a target outside the vocabulary
};

// The counted tokens in ascending order: their positions, targets and rows of
// hidden, padded.  For the gradients (dhidden not null) with zero rows behind up
// to a multiple of kDepth, and zeros into dhidden's rows of tokens that do not
// count.  Each workgroup finds its
// own tokens' places from the chunks before and its chunk's targets.
template <class In, class T>
__global__ __launch_bounds__(kRowBlock) void gather_kernel(const In* hidden, int64_t stride, int dim, Targets targets,
                                                           Selection out, T* h, int padded, int64_t plane, In* dhidden,
                                                           int64_t dstride) {
    __shared__ int32_t waves[kGathered];
    __shared__ int32_t any[kGathered];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kGathered, chunk = first / kChunkTokens;
    const int64_t end = first + kGathered < targets.tokens ? first + kGathered : targets.tokens;
    int32_t before = 0;  // counted tokens before the workgroup's first
    bool outside = false;
    for (int64_t k = threadIdx.x; k < chunk; k += kRowBlock) {
        const uint32_t c = out.chunks[k];
        before += static_cast<int32_t>(c & ~kOutside);
        outside |= (c & kOutside) != 0;
    }
    if (end > 0) {
        int64_t y[kChunkTokens / kRowBlock];
#pragma unroll
        for (int u = 0; u < kChunkTokens / kRowBlock; ++u) {
            const int64_t t = chunk * kChunkTokens + u * kRowBlock + threadIdx.x;
            y[u] = target_of(targets.ids, t < end ? t : end - 1);
        }
#pragma unroll
        for (int u = 0; u < kChunkTokens / kRowBlock; ++u) {
            const int64_t t = chunk * kChunkTokens + u * kRowBlock + threadIdx.x;
            before += t < first && targets.counts(y[u]);
            outside |= t < end && targets.outside(y[u]);
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) before += __shfl_xor(before, d);
    const uint64_t some = __ballot(outside);
    if (lane == 0) {
        waves[wave] = before;
        any[wave] = some != 0;
    }
    __syncthreads();
    before = 0;
    outside = false;
    for (int w = 0; w < kGathered; ++w) {
        before += waves[w];
        outside |= any[w] != 0;
    }
    uint32_t mine = 0;  // which of the workgroup's tokens count
    int64_t own = targets.ignored;
    for (int w = 0; w < kGathered; ++w) {
        const int64_t y = first + w < end ? target_of(targets.ids, first + w) : targets.ignored;
        mine |= static_cast<uint32_t>(targets.counts(y)) << w;
        if (w == wave) own = y;
    }
    const int64_t t = first + wave;
    if (mine >> wave & 1) {
        const int32_t at = before + __popc(mine & ((1u << wave) - 1));
        copy_row(hidden + t * stride, dim, h + static_cast<int64_t>(at) * padded, padded, plane, lane, 64);
        if (lane == 0) {
            out.rows[at] = static_cast<int32_t>(t);
            out.labels[at] = static_cast<int32_t>(own);
        }
    } else if (t < end) {
        if (lane == 0) out.losses[t] = own == targets.ignored ? 0.0f : __builtin_nanf("");
        if (dhidden) {
            constexpr int kVec = 16 / sizeof(In);
            In* row = dhidden + t * dstride;
            int c = lane * kVec;
            for (; c + kVec <= dim; c += 64 * kVec) *reinterpret_cast<Pack<In, kVec>*>(row + c) = Pack<In, kVec>{};
            for (; c < dim && c + kVec > dim; ++c) row[c] = static_cast<In>(0.0f);
        }
    }
    if (first + kGathered < targets.tokens) return;
    const int32_t n = before + __popc(mine);
    if (threadIdx.x == 0) {
        out.count[0] = n;
        out.count[1] = outside;
        out.count[2] = 0;
    }
    if (!dhidden) return;  // the scores do without the zero rows
    const int64_t rows = (static_cast<int64_t>(n) + kDepth - 1) / kDepth * kDepth;
    constexpr int kPlanes = sizeof(In) == 4 ? kSplitPlanes : 1;
    for (int q = 0; q < kPlanes; ++q) {
        Pack<T, 8>* zeros = reinterpret_cast<Pack<T, 8>*>(h + q * plane + static_cast<int64_t>(n) * padded);
        for (int64_t i = threadIdx.x; i < (rows - n) * padded / 8; i += kRowBlock) zeros[i] = Pack<T, 8>{};
    }
}

template <class In, class T>
__global__ __launch_bounds__(kRowBlock) void table_kernel(const In* table, int64_t stride, int dim, T* w, int padded,
                                                          int64_t plane) {
    copy_row(table + blockIdx.x * stride, dim, w + blockIdx.x * int64_t(padded), padded, plane, threadIdx.x, kRowBlock);
}

// ---------------------------------------------------------------------------
// scores: the first product, with the softmax's partial sums
// ---------------------------------------------------------------------------

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

// A block's logit gradients, none above 1, are held times this: binary16, whose
// smallest normal number is 2^-14 and whose range ends at 65504, keeps its full
// precision down to 2^-28 that way.
template <class E>
constexpr float kHeldUnit = 1.0f;
template <>
constexpr float kHeldUnit<f16> = 16384.0f;

// Until the normaliser is known a 16-bit type's exponentials exp2(-a), a >= 0,
// are held as codes of a: y = 2 + a * 30 / range lies in [2, 32), and the code
// is the last two bits of its exponent with the first 14 of its significand.
// Its step grows with a: exponentials above 2^-9 of the granule's maximum
// (binary16: above 1/6) are off by at most a twentieth (an eighth) of the
// type's unit roundoff, so the rounding of p - [label] to the products' type is
// the one that counts.  Exponentials rounded to that type, and p again
// behind them, are 0.5 to 1.5% less time for a call with gradients (16384 x
// 50257 x 2048 8.50 ms for 8.54), but the table gradient's rows without a label
// are then off by 3.37e-4 of their size for 2.89e-4 (180 tokens x 30522 x 1024,
// binary16; root mean square).  What lies below the range is zero in the type
// behind it, times kHeldUnit or not.
template <class E>
constexpr float kCodeRange = 136.0f;
template <>
constexpr float kCodeRange<f16> = 40.0f;
constexpr float kCodeFirst = 2.0f, kCodeSpan = 30.0f, kCodeLast = 31.9990234375f;
constexpr int kCodeShift = 9;

// below: -a, in powers of two.
template <class E>
__device__ __forceinline__ uint16_t code_of(float below) {
    const float y = __builtin_fmaf(below, -kCodeSpan / kCodeRange<E>, kCodeFirst);
    return static_cast<uint16_t>(__float_as_uint(fminf(y, kCodeLast)) >> kCodeShift);
}

// exp2(shift - a), a from the middle of the code's step.
template <class E>
__device__ __forceinline__ float exponential_of(uint16_t code, float shift) {
    const uint32_t half = 1u << (kCodeShift - 1), first = 0x40000000u;  // of kCodeFirst
    const float y = __uint_as_float(static_cast<uint32_t>(code) << kCodeShift | (first | half));
    return __builtin_amdgcn_exp2f(__builtin_fmaf(y, -kCodeRange<E> / kCodeSpan, shift + kCodeFirst * kCodeRange<E> / kCodeSpan));
}

struct ScoreOut {
    const int32_t* count;
    const int32_t* labels;
    int64_t first, block;      // the token block and B
    int64_t vocab, padded;
    float2* stats;
    float* label_logit;
    void* scores;              // null: the loss alone
    float* parts;              // a tile for each workgroup of the grid
    int64_t most_splits;       // parts that a tile's sum may be cut into
};

// A finished tile of scores, a wavefront's columns from the j0-th: each granule's
// maximum and sum, the labels' logits, and the exponentials into the block's
// scores (16-bit types: their codes).
template <class S, class E, int kColumns>
__device__ __forceinline__ void finish_scores(const ScoreOut& out, int64_t n, MICRO_SHARED char* area, const Place<S>& place,
                                              int64_t ta, int64_t tb, int j0, Acc (&acc)[S::kTilesA][kColumns]) {
    constexpr int kRun = 2;  // matrix tiles along a whose 16-bit values fill 128 bytes of a row
    const int64_t v0 = ta * S::kA + place.row(0, 0);
    // the wavefront's first row and token
    const int64_t w0 = ta * S::kA + place.wave_a, t0 = tb * S::kB + place.wave_b + j0 * 32;
    if ((ta + 1) * S::kA > out.vocab) {  // rows behind the vocabulary
        const int left = static_cast<int>(out.vocab - v0);
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const bool in = i * 32 + (r >> 2) * 8 + (r & 3) < left;
#pragma unroll
                for (int j = 0; j < kColumns; ++j) acc[i][j][r] = in ? acc[i][j][r] : -__builtin_inff();
            }
    }
#pragma unroll
    for (int j = 0; j < kColumns; ++j) {
        const int64_t token = tb * S::kB + place.column(j0 + j);
        const int64_t to_label = token < n ? out.labels[out.first + token] - v0 : -1;
        const int label = to_label >= 0 && to_label < S::kTilesA * 32 ? static_cast<int>(to_label) : -1;
        float most = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, acc[i][j][r]);
        if (__ballot(label >= 0) != 0) {  // few granules hold a label of the wavefront's tokens
            float at_label = 0.0f;
#pragma unroll
            for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    at_label = label == i * 32 + (r >> 2) * 8 + (r & 3) ? acc[i][j][r] : at_label;
            if (label >= 0 && (label & 4) == 0) out.label_logit[token] = at_label;
        }
        most = fmaxf(most, __shfl_xor(most, 32));
        // a granule without a finite maximum keeps its logits' own limits
        const float base = most == -__builtin_inff() ? 0.0f : most;
        float sum = 0.0f;
        const auto below = [base](float l) { return (l - base) * kLog2e; };
        if constexpr (sizeof(E) == 2) {
#pragma unroll
            for (int i = 0; i < S::kTilesA; i += kRun) {
#pragma unroll
                for (int m = 0; m < kRun && i + m < S::kTilesA; ++m)
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(below(acc[i + m][j][r]));
                if (out.scores) {
                    Chunk in[4], to[4];
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        if (i + m / 2 >= S::kTilesA) {
                            in[m] = Chunk{0, 0, 0, 0};
                            continue;
                        }
                        Vec4<uint16_t> lo, hi;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            lo[r] = code_of<E>(below(acc[i + m / 2][j][m % 2 * 8 + r]));
                            hi[r] = code_of<E>(below(acc[i + m / 2][j][m % 2 * 8 + 4 + r]));
                        }
                        swap_halves(lo, hi);
                        in[m] = __builtin_bit_cast(Chunk, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    }
                    exchange(area, in, to);
                    const int64_t v = w0 + i * 32 + (threadIdx.x & 7) * 8;
                    const bool in_tile = int(threadIdx.x & 7) * 8 < (S::kTilesA - i) * 32;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int64_t t = t0 + j * 32 + 8 * k + (threadIdx.x >> 3 & 7);
                        if (t < n && v < out.padded && in_tile)
                            *reinterpret_cast<Chunk*>(static_cast<E*>(out.scores) + t * out.padded + v) = to[k];
                    }
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < S::kTilesA; ++i) {
                Chunk in[4], to[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    Vec4<float> x;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        x[r] = __builtin_amdgcn_exp2f(below(acc[i][j][4 * q + r]));
                        sum += x[r];
                    }
                    in[q] = __builtin_bit_cast(Chunk, x);
                }
                if (out.scores) {
                    exchange(area, in, to);
                    const int64_t v = w0 + i * 32 + (threadIdx.x & 7) * 4;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int64_t t = t0 + j * 32 + 8 * k + (threadIdx.x >> 3 & 7);
                        if (t < n && v < out.padded)
                            *reinterpret_cast<Chunk*>(static_cast<E*>(out.scores) + t * out.padded + v) = to[k];
                    }
                }
            }
        }
        sum += __shfl_xor(sum, 32);
        if ((threadIdx.x & 32) == 0 && token < n) {
            const int64_t granule = v0 / (S::kTilesA * 32);
            out.stats[granule * out.block + token] = make_float2(most, sum);
        }
    }
}

// a: vocabulary, b: tokens, so a lane holds one token's logits and reduces
// them without shuffles but the one between its two halves.  Bound by the matrix
// cores: 16384 x 50257 x 2048 in 2.85 ms (1.18 PFLOP/s), of which the exponentials,
// their codes, maxima and stores of a finished tile are an eighth; alone, without
// scores to store, 8192 tokens in 1.27 to 1.39 ms (1.21 to 1.32).  Few tokens: by the one read of
// the table, 30 us for 206 MB (6.9 TB/s).  kCut: a short call over few tiles,
// whose tiles are cut along the sum and left for the join, since a step of one
// tile waits for its loads: whole calls of 7 tokens, 1549 x 2304, with gradients
// in 127 us for 237 (binary32, 101 since the gradients' parts count its six
// products' steps) and 58 for 66 (bfloat16).
template <class S, class T, class E, int kTerms, bool kCut>
__global__ __launch_bounds__(S::kThreads) void scores_kernel(Operand table, Operand h, int64_t blocks, ScoreOut out) {
    MICRO_STAGES(S);
    const int64_t counted = *out.count - out.first;
    const int64_t n = counted < out.block ? counted : out.block;
    if (n <= 0) return;
    h.kept = n;
    TileOrder order((out.vocab + S::kA - 1) / S::kA, (n + S::kB - 1) / S::kB, kCut ? out.most_splits : 1);
    Product<S, T, kTerms, false, false> product(table, h, blocks);
    const Place<S> place;
    MICRO_SHARED char* const area = stage1.a + (threadIdx.x >> 6) * kExchange;
    const int64_t steps = kTerms * blocks;
    const auto start = [&](const Tile& t) {
        if constexpr (kCut)
            product.start(t.a * S::kA, t.b * S::kB, steps * t.part / order.splits, steps * (t.part + 1) / order.splits, stage0);
        else
            product.start(t.a * S::kA, t.b * S::kB, 0, steps, stage0);
    };
    Tile tile, after;
    bool more = order.next(&tile);
    if (more) start(tile);
    for (; more; tile = after) {
        Acc acc[S::kTilesA][S::kTilesB];
        clear<S>(acc);
        product.run(acc, stage0, stage1);
        more = order.next(&after);
        if (more) start(after);
        if constexpr (kCut) {
#pragma unroll
            for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
                for (int j = 0; j < S::kTilesB; ++j) store_part<S>(tile_at<S>(out.parts, tile.index), i, j, acc[i][j]);
        } else {
            finish_scores<S, E, S::kTilesB>(out, n, area, place, tile.a, tile.b, 0, acc);
        }
    }
}

// Adds the parts of tiles whose sums were cut and finishes them.  A workgroup
// takes a column of matrix tiles of one wavefront; each of its own wavefronts
// adds every kJoinWaves-th part, the first one adds those sums, in their order.
constexpr int kJoinWaves = 4;
template <class S, class E>
__global__ __launch_bounds__(kJoinWaves * 64) void join_scores_kernel(ScoreOut out, int64_t grid) {
    __shared__ float sums[kJoinWaves - 1][S::kTilesA * 16][64];
    __shared__ __attribute__((aligned(1024))) char shared[kExchange];
    const int64_t counted = *out.count - out.first;
    const int64_t n = counted < out.block ? counted : out.block;
    if (n <= 0) return;
    const TileOrder order((out.vocab + S::kA - 1) / S::kA, (n + S::kB - 1) / S::kB, out.most_splits, grid);
    constexpr int kWaves = S::kThreads / 64;
    const int64_t t = blockIdx.x / (kWaves * S::kTilesB);
    if (t >= order.tail) return;
    const int of = blockIdx.x % (kWaves * S::kTilesB) / S::kTilesB, j = blockIdx.x % S::kTilesB;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int64_t ta, tb;
    order.place(t, &ta, &tb);
    const Place<S> place(of);
    if (tb * S::kB + place.wave_b + j * 32 >= n) return;
    Acc acc[S::kTilesA][1];
#pragma unroll
    for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][0][r] = 0.0f;
#pragma unroll 2
    for (int64_t s = wave; s < order.splits; s += kJoinWaves)
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i) add_part<S>(tile_at<S>(out.parts, s * order.tail + t, of * 64 + lane), i, j, acc[i][0]);
#pragma unroll
    for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (wave > 0) sums[wave - 1][i * 16 + r][lane] = acc[i][0][r];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < kJoinWaves - 1; ++w)
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][0][r] += sums[w][i * 16 + r][lane];
    finish_scores<S, E, 1>(out, n, (MICRO_SHARED char*)shared, place, ta, tb, j, acc);
}

// ---------------------------------------------------------------------------
// between the products
// ---------------------------------------------------------------------------

// The sum or mean of the counted tokens' losses, in binary64 and an order that
// only their number and the workgroup's size determine; NaN when a target lies
// outside the vocabulary.
template <int kThreads>
__device__ void total_loss(const int32_t* count, const float* losses, bool mean, float* loss) {
    constexpr int kEach = 8;
    __shared__ double waves[kThreads / 64];
    const int64_t n = count[0];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kEach * kThreads) {
        float x[kEach];
#pragma unroll
        for (int u = 0; u < kEach; ++u)
            x[u] = __hip_atomic_load(losses + (i + u * kThreads < n ? i + u * kThreads : n - 1), __ATOMIC_RELAXED,
                                     __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int u = 0; u < kEach; ++u)
            if (i + u * kThreads < n) sum += static_cast<double>(x[u]);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x != 0) return;
    sum = 0.0;
    for (int w = 0; w < kThreads / 64; ++w) sum += waves[w];
    if (count[1]) sum = __builtin_nan("");
    *loss = static_cast<float>(mean && n > 0 ? sum / static_cast<double>(n) : sum);
}

constexpr int kJoinAhead = 8;
constexpr int64_t kFewJoined = 2048;

// Maximum, inverse sum and loss of every counted token of the block, from its
// granules: kTokens tokens a workgroup, kSlices threads each.
// loss (not null where these are all tokens and few workgroups): the workgroup
// that finishes last adds the losses up.
template <int kTokens, int kSlices>
__global__ __launch_bounds__(kTokens* kSlices) void softmax_kernel(int32_t* count, int64_t first, int64_t block,
                                                                   const float2* stats, int64_t granules,
                                                                   const float* label_logit, const int32_t* rows,
                                                                   float2* softmax, float* counted_losses, float* losses,
                                                                   bool mean, float* loss) {
    __shared__ float2 part[kSlices][kTokens];
    const int64_t counted = *count - first, n = counted < block ? counted : block;
    const int64_t token = static_cast<int64_t>(blockIdx.x) * kTokens + (threadIdx.x % kTokens);
    const int slice = threadIdx.x / kTokens;
    if (static_cast<int64_t>(blockIdx.x) * kTokens >= (n > 0 || !loss ? n : 1)) return;
    if (n <= 0) {  // nothing counts: the first workgroup says so
        total_loss<kTokens * kSlices>(count, counted_losses, mean, loss);
        return;
    }
    const int64_t at = token < n ? token : n - 1;
    float most = -__builtin_inff(), sum = 0.0f;
    const auto join = [&](const auto& s, int parts) {
        float to = most;
#pragma unroll
        for (int u = 0; u < parts; ++u) to = fmaxf(to, s[u].x);
        // of granules without any finite maximum the sums are 0, or NaN
        const float base = to == -__builtin_inff() ? 0.0f : to;
        sum *= __builtin_amdgcn_exp2f((most == to ? 0.0f : most - base) * kLog2e);
#pragma unroll
        for (int u = 0; u < parts; ++u) sum += s[u].y * __builtin_amdgcn_exp2f((s[u].x == to ? 0.0f : s[u].x - base) * kLog2e);
        most = to;
    };
    const auto finish_token = [&] {
        // (the label's logit is often the maximum itself, and their difference exact)
        const float own = (most - label_logit[token]) + logf(sum);
        softmax[token] = make_float2(most, 1.0f / sum);
        __hip_atomic_store(counted_losses + first + token, own, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        losses[rows[first + token]] = own;
    };
    for (int64_t g = slice; g < granules; g += kJoinAhead * kSlices) {
        float2 s[kJoinAhead];
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
            s[u] = stats[(g + u * kSlices < granules ? g + u * kSlices : granules - 1) * block + at];
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u)
            if (g + u * kSlices >= granules) s[u] = make_float2(-__builtin_inff(), 0.0f);
        join(s, kJoinAhead);
    }
    part[slice][threadIdx.x % kTokens] = make_float2(most, sum);
    for (int half = kSlices / 2; half > 0; half /= 2) {
        __syncthreads();
        if (slice < half) {
            const float2 other[1] = {part[slice + half][threadIdx.x % kTokens]};
            join(other, 1);
            part[slice][threadIdx.x % kTokens] = make_float2(most, sum);
        }
    }
    if (slice == 0 && token < n) finish_token();
    if (!loss) return;
    // the losses of this workgroup, then its arrival
    __shared__ bool last;
    __syncthreads();
    if (threadIdx.x == 0) {
        const int32_t groups = static_cast<int32_t>((n + kTokens - 1) / kTokens);
        last = __hip_atomic_fetch_add(count + 2, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == groups - 1;
    }
    __syncthreads();
    if (last) total_loss<kTokens * kSlices>(count, counted_losses, mean, loss);
}

constexpr int kTurnBlock = 256, kTurnRows = 16;

// The exponentials of a block become the logit gradients, in place (binary32:
// into three planes): times exp(granule's maximum - lse), less one at the
// label, rounded to the products' type.  There p - 1 comes from the token's
// binary32 loss, so a token that is nearly certain keeps its small gradient, and
// what its rounding leaves goes into label_rest.  Zero rows up to a multiple
// of kDepth.  A stream of one read and one write of the block's scores, bound by
// HBM: 3.3 GB in 625 us (5.3 TB/s).
template <class E, class T>
__global__ __launch_bounds__(kTurnBlock) void gradient_kernel(const int32_t* count, int64_t first, int64_t block, E* scores,
                                                              int64_t padded, const float2* stats, int granule,
                                                              const float2* softmax, const float* counted_losses,
                                                              const int32_t* labels, T* split, float* label_rest) {
    constexpr int kVec = 16 / sizeof(E);
    const int64_t counted = *count - first, n = counted < block ? counted : block;
    if (n <= 0) return;
    const int64_t rows = (n + kDepth - 1) / kDepth * kDepth, plane = block * padded;
    const int64_t v = (static_cast<int64_t>(blockIdx.x) * kTurnBlock + threadIdx.x) * kVec;
    if (v >= padded) return;
    const int64_t g = v / granule;
    for (int64_t token = static_cast<int64_t>(blockIdx.y) * kTurnRows; token < rows;
         token += static_cast<int64_t>(gridDim.y) * kTurnRows)
#pragma unroll 4
        for (int u = 0; u < kTurnRows; ++u) {
            const int64_t t = token + u;
            if (t >= rows) break;
            E* at = scores + t * padded + v;
            float x[kVec] = {};
            if (t < n) {
                const float2 of = softmax[t];
                const float below = (stats[g * block + t].x - of.x) * kLog2e;  // the granule's maximum
                const int64_t label = labels[first + t] - v;
                if constexpr (sizeof(E) == 4) {
                    load_floats<E, kVec>(at, x);
                    const float factor = of.y * __builtin_amdgcn_exp2f(below);
#pragma unroll
                    for (int j = 0; j < kVec; ++j) x[j] *= factor;
                } else {
                    const Pack<uint16_t, kVec> codes = *reinterpret_cast<const Pack<uint16_t, kVec>*>(at);
                    const float shift = below + __builtin_amdgcn_logf(of.y * kHeldUnit<E>);
#pragma unroll
                    for (int j = 0; j < kVec; ++j) x[j] = exponential_of<E>(codes.v[j], shift);
                }
                if (label >= 0 && label < kVec) {
                    const float p = kHeldUnit<E> * expm1f(-counted_losses[first + t]);
                    if constexpr (sizeof(E) == 2) label_rest[t] = p - static_cast<float>(rounded<E>(p));
#pragma unroll
                    for (int j = 0; j < kVec; ++j)
                        if (label == j) x[j] = p;
                }
            }
            if constexpr (sizeof(E) == 4) {
                Pack<T, kVec> p[kSplitPlanes];
#pragma unroll
                for (int j = 0; j < kVec; ++j) split3(x[j], p[0].v[j], p[1].v[j], p[2].v[j]);
#pragma unroll
                for (int q = 0; q < kSplitPlanes; ++q)
                    *reinterpret_cast<Pack<T, kVec>*>(split + q * plane + t * padded + v) = p[q];
            } else {
                store_floats<E, kVec>(at, x);
            }
        }
}

// ---------------------------------------------------------------------------
// the gradients: the second and third product
// ---------------------------------------------------------------------------

struct GradientOut {
    const int32_t* count;
    int64_t first, block;      // of the token block
    bool table;                // dtable (b: vocabulary, k: tokens), else dhidden (b: tokens, k: vocabulary)
    int64_t vocab;
    int32_t dim;
    const int32_t* rows;
    float scale;
    bool mean;
    float unit;                // kHeldUnit
    void* to;                  // output rows
    int64_t stride;
    bool accumulate;
    float* partials;           // one tile a workgroup of the grid
    float* carried;
    int terms;                 // of the products
    // dhidden of 16-bit types: p - 1 at the label less its rounding, and the
    // table's rows as the product reads them
    const float* label_rest;
    const int32_t* labels;
    const void* table_rows;
    int64_t table_stride;
};

struct GradientPlan {
    int64_t n;          // tokens of the block
    int64_t tiles_a, tiles_b, blocks;
    int64_t most_splits;
    bool last;          // no token block after this one
};

// The same on every workgroup of the product and of its join.
template <class S>
__device__ GradientPlan gradient_plan(const GradientOut& o) {
    GradientPlan p;
    const int64_t counted = *o.count - o.first;
    p.n = counted < 0 ? 0 : counted < o.block ? counted : o.block;
    p.last = counted <= o.block;
    const int64_t columns = o.table ? o.vocab : p.n;
    p.tiles_a = (o.dim + S::kA - 1) / S::kA;
    p.tiles_b = (columns + S::kB - 1) / S::kB;
    p.blocks = ((o.table ? p.n : o.vocab) + kDepth - 1) / kDepth;
    p.most_splits = o.terms * p.blocks / 8;  // a part of fewer steps is not worth its partial tile
    return p;
}

// A token block with nothing counted leaves the table's gradient to the block
// before it; the first block always writes.
__device__ __forceinline__ bool nothing_to_do(const GradientOut& o, const GradientPlan& p) {
    return p.n == 0 && (!o.table || o.first > 0);
}

// The factor of both gradients.
__device__ __forceinline__ float gradient_factor(const GradientOut& o) {
    const int32_t all = *o.count;
    return (o.mean ? (all > 0 ? o.scale / static_cast<float>(all) : 0.0f) : o.scale) / o.unit;
}

// A finished tile: into the carried sums while token blocks follow, else scaled
// and rounded into the output.  16-bit values change hands rounded, two matrix
// tiles along a at a time; binary32 ones, and those that are added to, in 32
// bits.
template <class S, class Out, int kParts>
__device__ __forceinline__ void finish(const GradientOut& o, const GradientPlan& p, MICRO_SHARED char* area, int64_t ta,
                                       int64_t tb, int i0, int j, Acc (&acc)[kParts]) {
    if (o.table && o.first > 0)
#pragma unroll
        for (int i = 0; i < kParts; ++i) add_part<S>(tile_at<S>(o.carried, tb * p.tiles_a + ta), i0 + i, j, acc[i]);
    if (o.table && !p.last) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) store_part<S>(tile_at<S>(o.carried, tb * p.tiles_a + ta), i0 + i, j, acc[i]);
        return;
    }
    const float factor = gradient_factor(o);
    const Place<S> place;
    const int64_t columns = o.table ? o.vocab : p.n;
    const int64_t b0 = tb * S::kB + place.wave_b + j * 32 + (threadIdx.x >> 3 & 7);
    const int64_t a0 = ta * S::kA + place.wave_a + i0 * 32;
    Chunk in[4], to[4];
    const auto row = [&](int k) -> Out* {
        const int64_t b = b0 + 8 * k;
        if (b >= columns) return nullptr;
        return static_cast<Out*>(o.to) + (o.table ? b : o.rows[o.first + b]) * o.stride;
    };
    if constexpr (sizeof(Out) == 2) {
        if (!o.accumulate) {
#pragma unroll
            for (int i = 0; i < kParts; i += 2) {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    Vec4<Out> lo{}, hi{};
                    if (i + m / 2 < kParts) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            lo[r] = rounded<Out>(factor * acc[i + m / 2][m % 2 * 8 + r]);
                            hi[r] = rounded<Out>(factor * acc[i + m / 2][m % 2 * 8 + 4 + r]);
                        }
                    }
                    swap_halves(lo, hi);
                    in[m] = __builtin_bit_cast(Chunk, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                }
                exchange(area, in, to);
                const int64_t a = a0 + i * 32 + (threadIdx.x & 7) * 8;
                if ((threadIdx.x & 4) != 0 && i + 1 >= kParts) continue;  // the second matrix tile is not there
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    Out* at = row(k);
                    if (!at) break;
                    const Pack<Out, 8> x = __builtin_bit_cast(Pack<Out, 8>, to[k]);
                    if (a + 8 <= o.dim) {
                        *reinterpret_cast<Pack<Out, 8>*>(at + a) = x;
                    } else {
#pragma unroll
                        for (int r = 0; r < 8; ++r)
                            if (a + r < o.dim) at[a + r] = x.v[r];
                    }
                }
            }
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            in[q] = __builtin_bit_cast(Chunk, Vec4<float>{acc[i][4 * q], acc[i][4 * q + 1], acc[i][4 * q + 2], acc[i][4 * q + 3]});
        exchange(area, in, to);
        const int64_t a = a0 + i * 32 + (threadIdx.x & 7) * 4;
        if (a >= o.dim) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            Out* at = row(k);
            if (!at) break;
            at += a;
            const Vec4<float> sums = __builtin_bit_cast(Vec4<float>, to[k]);
            float x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = factor * sums[r];
            if (a + 4 <= o.dim) {
                if (o.accumulate) {
                    float old[4];
                    load_floats<Out, 4>(at, old);
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] += old[r];
                }
                store_floats<Out, 4>(at, x);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (a + r < o.dim) at[r] = rounded<Out>(o.accumulate ? static_cast<float>(at[r]) + x[r] : x[r]);
            }
        }
    }
}

// Adds the parts of the tiles that were cut, in their order; a workgroup a 32 x
// 32 part of each wavefront's, so that a few tiles occupy many.  grid: of the
// product.
template <class S, class Out>
__device__ __forceinline__ void join_parts(const GradientOut& o, int64_t grid, MICRO_SHARED char* area) {
    const GradientPlan p = gradient_plan<S>(o);
    if (nothing_to_do(o, p)) return;
    const TileOrder order(p.tiles_a, p.tiles_b, p.most_splits, grid);
    if (order.splits == 1) return;
    constexpr int kParts = S::kTilesA * S::kTilesB;
    for (int64_t u = blockIdx.x; u < order.tail * kParts; u += gridDim.x) {
        const int64_t t = u / kParts;
        const int i = static_cast<int>(u % kParts) / S::kTilesB, j = static_cast<int>(u % kParts) % S::kTilesB;
        Acc acc[1];
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[0][r] = 0.0f;
#pragma unroll 4
        for (int64_t s = 0; s < order.splits; ++s) add_part<S>(tile_at<S>(o.partials, s * order.tail + t), i, j, acc[0]);
        int64_t ta, tb;
        order.place(order.full + t, &ta, &tb);
        finish<S, Out, 1>(o, p, area, ta, tb, i, j, acc);
    }
}

// What dhidden's tile starts from: the label's term, by far the largest of a
// token, gets back what the rounding of its operand took.  So dhidden is off by
// what its own rounding takes alone (4915 x 30522 x 1024 bfloat16: 1.66e-3 of its
// size in root mean square; 1.97e-3 without).  Here rather than when the tile is
// finished: the first stage's loads are under way, and registers are free (there
// they were not: 300 bytes a lane went to scratch, and the call took 5% longer).
template <class S, class T>
__device__ __forceinline__ void label_rests(const GradientOut& o, const GradientPlan& p, int64_t ta, int64_t tb,
                                            Acc (&acc)[S::kTilesA][S::kTilesB]) {
    const Place<S> place;
    const int64_t a = ta * S::kA + place.row(0, 0);
    const int left = static_cast<int>(o.dim - a);  // (rows are padded to whole runs of four)
#pragma unroll
    for (int j = 0; j < S::kTilesB; ++j) {
        const int64_t token = tb * S::kB + place.column(j);
        const float rest = token < p.n ? o.label_rest[token] : 0.0f;
        const T* row = static_cast<const T*>(o.table_rows) + (token < p.n ? o.labels[o.first + token] : 0) * o.table_stride + a;
#pragma unroll
        for (int i = 0; i < S::kTilesA; ++i) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float w[4] = {};
                if (rest != 0.0f && i * 32 + q * 8 < left) load_floats<T, 4>(row + (i * 32 + q * 8), w);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][4 * q + r] = rest * w[r];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// kTable: dtable^T = h^T g, else dhidden^T = W^T g^T.  a is always the width,
// so a lane's values are adjacent in an output row.  Bound by the matrix cores:
// 16384 x 50257 x 2048 in 2.6 and 2.55 ms (1.29 and 1.32 PFLOP/s).  dhidden's
// split tiles, if any, are joined here by the workgroups of dtable's product,
// which saves a launch.
template <class S, class T, class Out, int kTerms, bool kTable>
__global__ __launch_bounds__(S::kThreads) void gradients_kernel(Operand wide, Operand g, GradientOut o, GradientOut hidden) {
    MICRO_STAGES(S);
    if (kTable) join_parts<S, Out>(hidden, gridDim.x, stage1.a + (threadIdx.x >> 6) * kExchange);
    const GradientPlan p = gradient_plan<S>(o);
    if (nothing_to_do(o, p)) return;
    if (kTable) {
        wide.depth = g.depth = p.blocks * kDepth;  // zero rows behind the last token
    } else {
        g.kept = p.n;
    }
    TileOrder order(p.tiles_a, p.tiles_b, p.most_splits);
    Product<S, T, kTerms, true, kTable> product(wide, g, p.blocks);
    const int64_t steps = kTerms * p.blocks;
    MICRO_SHARED char* const area = stage1.a + (threadIdx.x >> 6) * kExchange;
    const auto start = [&](const Tile& t) {
        product.start(t.a * S::kA, t.b * S::kB, t.part < 0 ? 0 : steps * t.part / order.splits,
                      t.part < 0 ? steps : steps * (t.part + 1) / order.splits, stage0);
    };
    Tile tile, after;
    bool more = order.next(&tile);
    if (more) start(tile);
    for (; more; tile = after) {
        Acc acc[S::kTilesA][S::kTilesB];
        clear<S>(acc);
        if constexpr (!kTable && sizeof(Out) == 2)
            if (tile.part <= 0) label_rests<S, T>(o, p, tile.a, tile.b, acc);
        product.run(acc, stage0, stage1);
        more = order.next(&after);
        if (more) start(after);
#pragma unroll
        for (int j = 0; j < S::kTilesB; ++j) {
            Acc column[S::kTilesA];
#pragma unroll
            for (int i = 0; i < S::kTilesA; ++i) column[i] = acc[i][j];
            if (tile.part < 0) {
                finish<S, Out, S::kTilesA>(o, p, area, tile.a, tile.b, 0, j, column);
            } else {
#pragma unroll
                for (int i = 0; i < S::kTilesA; ++i) store_part<S>(tile_at<S>(o.partials, tile.index), i, j, column[i]);
            }
        }
    }
}

template <class S, class Out>
__global__ __launch_bounds__(S::kThreads) void join_parts_kernel(GradientOut o, int grid) {
    __shared__ __attribute__((aligned(1024))) char shared[S::kThreads / 64 * kExchange];
    join_parts<S, Out>(o, grid, (MICRO_SHARED char*)shared + (threadIdx.x >> 6) * kExchange);
}

constexpr int kTotalBlock = 1024;

__global__ __launch_bounds__(kTotalBlock) void total_kernel(const int32_t* count, const float* losses, bool mean, float* loss) {
    total_loss<kTotalBlock>(count, losses, mean, loss);
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

// The score product of a short call is cut along its sum where its tiles are no
// more than this part of the grid, kCutSteps steps a part at least.  (A quarter
// of the grid, or parts of 4 steps: the join's launch then costs what it saves,
// 22 us for 19 at 20 tokens, 7000 x 768; 61 for 58 at 300, 1600 x 512.)
constexpr int kFewTiles = 8, kCutSteps = 8;

uint32_t ceil_div(int64_t a, int64_t b) { return static_cast<uint32_t>((a + b - 1) / b); }

template <class S>
int product_grid(const LossCall& c) {
    return c.compute_units * S::kPerUnit / TileOrder::kDies * TileOrder::kDies;
}

// In: the tensors' type; T: the products'; E: the scores' (16 bits: codes of the
// exponentials, then logit gradients); S: the tiles.
template <class In, class T, class E, int kTerms, class S>
hipError_t run(const LossCall& c, hipStream_t stream) {
    constexpr bool kSplit = sizeof(In) == 4;
    const int64_t rows_h = (std::max<int64_t>(c.tokens, 1) + kDepth - 1) / kDepth * kDepth;
    const Targets targets{c.targets, c.tokens, c.ignored, c.vocab};
    hipError_t e = hipSuccess;
    if (c.tokens > kChunkTokens)
        e = launch(count_kernel, dim3(ceil_div(c.tokens, kChunkTokens)), dim3(kChunkTokens), stream, targets, c.chunks);
    if (e != hipSuccess) return e;
    e = launch(gather_kernel<In, T>, dim3(ceil_div(std::max<int64_t>(c.tokens, 1), kGathered)), dim3(kRowBlock), stream,
               static_cast<const In*>(c.hidden.at), c.hidden.stride, c.dim, targets,
               Selection{c.chunks, c.count, c.rows, c.labels, c.losses}, static_cast<T*>(c.h), c.dim_padded,
               rows_h * c.dim_padded, c.gradients ? static_cast<In*>(c.dhidden.at) : nullptr, c.dhidden.stride);
    if (e != hipSuccess) return e;
    Operand table{c.table.at, c.table.stride, c.vocab, 0, 0};
    if (!table_in_place(c)) {
        table = {c.w, c.dim_padded, c.vocab, 0, c.vocab * c.dim_padded};
        e = launch(table_kernel<In, T>, dim3(static_cast<uint32_t>(c.vocab)), dim3(kRowBlock), stream,
                   static_cast<const In*>(c.table.at), c.table.stride, c.dim, static_cast<T*>(c.w), c.dim_padded, table.plane);
        if (e != hipSuccess) return e;
    }
    const int granule = S::kTilesA * 32;
    // a call of few tokens has more granules, and room for them in a shorter block
    const int64_t block = granule == kGranuleFew ? kFewTokens : granule == kGranuleSome ? std::min<int64_t>(kSomeTokens, c.block) : c.block;
    const int64_t granules = (c.vocab + S::kA - 1) / S::kA * S::kWavesA;
    const int grid = product_grid<S>(c);
    const int64_t blocks = c.dim_padded / kDepth, steps = kTerms * blocks;
    bool total_now = false;
    for (int64_t first = 0; first < c.tokens || first == 0; first += block) {
        const int64_t most = std::max<int64_t>(std::min(c.tokens - first, block), 1);
        const Operand h{static_cast<const T*>(c.h) + first * c.dim_padded, c.dim_padded, 0, 0, rows_h * c.dim_padded};
        const ScoreOut scores{c.count, c.labels, first, block, c.vocab, c.vocab_padded, c.stats, c.label_logit,
                              c.gradients ? c.scores : nullptr, c.parts, steps / kCutSteps};
        const int64_t tiles = int64_t(ceil_div(c.vocab, S::kA)) * ceil_div(most, S::kB);
        bool cut = false;
        if constexpr (S::kA * S::kB <= kPartTile) {
            static_assert(S::kPerUnit * S::kA * S::kB <= 2 * kPartTile, "a part for each workgroup");
            cut = scores.most_splits > 1 && tiles <= grid / kFewTiles;
            if (cut) {
                e = launch(scores_kernel<S, T, E, kTerms, true>, dim3(grid), dim3(S::kThreads), stream, table, h, blocks,
                           scores);
                if (e != hipSuccess) return e;
                e = launch(join_scores_kernel<S, E>, dim3(static_cast<uint32_t>(tiles * (S::kThreads / 64) * S::kTilesB)),
                           dim3(kJoinWaves * 64), stream, scores, int64_t(grid));
            }
        }
        if (!cut)
            e = launch(scores_kernel<S, T, E, kTerms, false>, dim3(grid), dim3(S::kThreads), stream, table, h, blocks, scores);
        if (e != hipSuccess) return e;
        total_now = c.tokens <= std::min<int64_t>(block, kSomeTokens);
        const auto join = [&](auto kernel, int tokens, int slices) {
            return launch(kernel, dim3(ceil_div(most, tokens)), dim3(tokens * slices), stream, c.count, first, block, c.stats,
                          granules, c.label_logit, c.rows, c.softmax, c.counted_losses, c.losses, c.mean,
                          total_now ? c.loss : nullptr);
        };
        // few tokens: more threads for each, so that enough loads are under way
        e = most <= kFewJoined ? join(softmax_kernel<8, 128>, 8, 128) : join(softmax_kernel<32, 16>, 32, 16);
        if (e != hipSuccess) return e;
        if (!c.gradients) continue;
        const uint32_t turns = ceil_div(c.vocab_padded, kTurnBlock * (16 / int(sizeof(E))));
        // (a grid's second dimension ends at 65535; the kernel goes on by its size)
        const uint32_t turn_rows = std::min<uint32_t>(ceil_div((most + kDepth - 1) / kDepth * kDepth, kTurnRows), 32768);
        e = launch(gradient_kernel<E, T>, dim3(turns, turn_rows), dim3(kTurnBlock), stream, c.count, first, block,
                   static_cast<E*>(c.scores), c.vocab_padded, c.stats, granule, c.softmax, c.counted_losses, c.labels,
                   static_cast<T*>(c.split), c.label_rest);
        if (e != hipSuccess) return e;
        // g as the operand of both products
        Operand g{kSplit ? c.split : c.scores, c.vocab_padded, 0, 0, block * c.vocab_padded};
        GradientOut o{c.count, first, block, false, c.vocab, c.dim, c.rows, c.scale, c.mean, kHeldUnit<T>,
                      c.dhidden.at, c.dhidden.stride, false, c.partials, c.carried, kTerms,
                      c.label_rest, c.labels, table.at, table.stride};
        Operand wide{table.at, table.stride, c.dim_padded, c.vocab, table.plane};
        e = launch(gradients_kernel<S, T, In, kTerms, false>, dim3(grid), dim3(S::kThreads), stream, wide, g, o, o);
        if (e != hipSuccess) return e;
        const GradientOut of_hidden = o;  // its split tiles are joined by the next product's workgroups
        o.table = true;
        o.to = c.dtable.at;
        o.stride = c.dtable.stride;
        o.accumulate = c.accumulate;
        o.partials += c.compute_units * kWideTile;
        wide = {h.at, h.stride, c.dim_padded, 0, h.plane};
        g.kept = c.vocab_padded;
        e = launch(gradients_kernel<S, T, In, kTerms, true>, dim3(grid), dim3(S::kThreads), stream, wide, g, o, of_hidden);
        if (e != hipSuccess) return e;
        e = launch(join_parts_kernel<S, In>, dim3(grid), dim3(S::kThreads), stream, o, grid);
        if (e != hipSuccess) return e;
    }
    if (total_now) return hipSuccess;
    return launch(total_kernel, dim3(1), dim3(kTotalBlock), stream, c.count, c.counted_losses, c.mean, c.loss);
}

template <class In, class T, class E, int kTerms>
hipError_t pick(const LossCall& c, hipStream_t stream) {
    if (c.tokens <= kFewTokens && !c.gradients) return run<In, T, E, kTerms, Narrow32>(c, stream);
    if (c.tokens <= kSomeTokens) return run<In, T, E, kTerms, Middle>(c, stream);
    return run<In, T, E, kTerms, Wide>(c, stream);
}

}  // namespace

// 16-byte loads of whole steps of kDepth values.
bool table_in_place(const LossCall& c) {
    return c.type != MICRO_TYPE_F32 && c.dim % kDepth == 0 && c.table.stride % 8 == 0 &&
           reinterpret_cast<uintptr_t>(c.table.at) % 16 == 0 && c.table.stride < (int64_t(1) << 22);
}

hipError_t launch_loss(const LossCall& c, hipStream_t stream) {
    if (c.type == MICRO_TYPE_F32) return pick<float, bf16, float, 6>(c, stream);
    if (c.type == MICRO_TYPE_F16) return pick<f16, f16, f16, 1>(c, stream);
    return pick<bf16, bf16, bf16, 1>(c, stream);
}

}  // namespace micro

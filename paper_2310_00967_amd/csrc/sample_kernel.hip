// gfx950 kernel that draws a token from each row of logits:
//   m = max l,   w_i = exp((l_i - m) / T),   ordered by (logit descending, index)
//   kept: the first top_k, of those the shortest prefix that reaches top_p of
//   their weight, of those w_i >= min_p
//   token: the first index where the running sum of kept weights exceeds u times
//   their sum
// Weights are computed in binary64 and rounded to whole multiples of 2^-f; their
// sums are of 64-bit integers and exact, so the token does not depend on how a row
// is divided, and a border between two tokens lies where binary64 sums have it
// to 2^-f.
//
// A workgroup takes a row and reads it again for each step (from the second time on out
// of the caches).  A small top_k needs two readings: the k-th largest of the threads'
// maxima is a lower bound of the k-th logit, and the few logits above it are sorted in
// shared memory, where all else follows.  Else the weights are added into bins that
// divide the range of logits that weigh anything, which finds the bin where top_p cuts;
// its few logits are sorted; a third reading adds what is kept by the wavefronts' runs of
// indices; and the run that holds the token is walked.  A cut that these lists do not
// hold (thousands of equal logits) and a large top_k are found by histograms over the
// logits' bits.
#include "sample_kernel.h"

#include "launch.h"
#include "value_types.h"

namespace micro {
namespace {

constexpr int kBins = 4096, kKeyBits = 12;  // 2^kKeyBits of them for a level over keys
constexpr int kBatches = 4096;              // of a row, at most
constexpr int kExpSteps = 64;               // of the table of 2^(j / 64)
constexpr float kLowest = -3.40282346638528859812e+38f;

// Bits of a logit in its order: larger logits have larger keys, -0 and 0 the same.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t key) {
    return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu));
}

// floor(f * x) and ceil(f * x) of a binary64 f in [0, 1], exactly.
__device__ __forceinline__ uint64_t share_of(double f, uint64_t x, bool up) {
    if (!(f > 0.0)) return 0;
    if (f >= 1.0) return x;
    const uint64_t bits = __builtin_bit_cast(uint64_t, f);
    const int exponent = static_cast<int>(bits >> 52);  // f = mantissa * 2^(exponent - 1075)
    if (exponent == 0) return up && x > 0 ? 1 : 0;      // below 2^-1022: less than one of 2^63
    const uint64_t mantissa = (bits & ((uint64_t(1) << 52) - 1)) | (uint64_t(1) << 52);
    const uint64_t lo = mantissa * x, hi = __umul64hi(mantissa, x);
    const int shift = 1075 - exponent;  // 53 and more
    uint64_t whole = 0;
    bool rest;
    if (shift < 64) {
        whole = hi << (64 - shift) | lo >> shift;
        rest = (lo << (64 - shift)) != 0;
    } else if (shift < 128) {
        whole = shift == 64 ? hi : hi >> (shift - 64);
        rest = lo != 0 || (shift > 64 && (hi << (128 - shift)) != 0);
    } else {
        rest = (hi | lo) != 0;
    }
    return whole + (up && rest ? 1 : 0);
}

// kThreads: of a workgroup, and entries of a sorted list; up to kThreads / 2 is a top_k
// small enough for lists.
template <int kThreads>
struct Shared {
    static constexpr int kWaves = kThreads / 64, kList = kThreads;
    double powers[kExpSteps];
    uint64_t bins[kBins];
    uint64_t batches[kBatches];  // sums over runs of indices
    uint64_t list[kList];
    uint64_t waves[kWaves];
    uint64_t value, before;  // one thread's answer to all
    uint32_t chosen, count;
};

// Weights of one row.
struct Weigher {
    const double* powers;
    double most, steps;  // steps: of 1 / 64 of a power of two in a unit of logit
    double least;        // in steps; what is below weighs nothing
    int32_t unit;        // 2^bits in a binary64's upper word

    // exp(y) 2^bits to the nearest integer, y = (x - m) / T, by a table of 2^(j/64) and
    // a polynomial of the rest, below h = 2^-7.5: its series with the fifth power
    // replaced by lower ones (r^5 ~ 5/4 h^2 r^3 - 5/16 h^4 r), which is off by h^5 / 1920
    // = 2.4e-15.  (The table as in Tang's method, 1989.)
    // As `kBias` plus the integer.
    static constexpr uint64_t kBias = uint64_t(0x433) << 52;
    __device__ __forceinline__ uint64_t biased(float x) const {
        constexpr double kStep = 0.6931471805599453 / kExpSteps, h = kStep / 2;
        constexpr double c1 = (1.0 - h * h * h * h / 384) * kStep, c2 = 0.5 * kStep * kStep;
        constexpr double c3 = (1.0 / 6 + h * h / 96) * kStep * kStep * kStep, c4 = kStep * kStep * kStep * kStep / 24;
        constexpr double kRound = 6755399441055744.0;  // 1.5 * 2^52: the integer is left in the last bits
        // (also where a masked logit times a step of 0 is no number)
        const double t = __builtin_fmax((static_cast<double>(x) - most) * steps, least);
        const double n = t + kRound;
        const double r = t - (n - kRound);
        const int32_t i = static_cast<int32_t>(__builtin_bit_cast(uint64_t, n));
        double s = __builtin_fma(r, c4, c3);
        s = __builtin_fma(r, s, c2);
        s = __builtin_fma(r, s, c1);
        s = __builtin_fma(r, s, 1.0);
        const uint64_t p = __builtin_bit_cast(uint64_t, powers[i & (kExpSteps - 1)]);
        const uint32_t upper = static_cast<uint32_t>(p >> 32) + ((i >> 6) << 20) + unit;
        const double scaled = __builtin_bit_cast(double, static_cast<uint64_t>(upper) << 32 | static_cast<uint32_t>(p));
        const double sum = __builtin_fma(s, scaled, 4503599627370496.0);
        return __builtin_bit_cast(uint64_t, sum);
    }
    __device__ __forceinline__ uint64_t weight(float x) const { return biased(x) - kBias; }
    __device__ __forceinline__ double exponent(float x) const {
        return (static_cast<double>(x) - most) * (steps * (0.6931471805599453 / kExpSteps));
    }
};

// The kept prefix of the order: logits from `low` up, and of those that equal `at`, just
// below `low`, the ones up to index `last` (at = low: there are no such).
struct Cut {
    float low, at;
    uint32_t last;
    __device__ __forceinline__ explicit Cut(float from) : low(from), at(from), last(0) {}
    __device__ __forceinline__ Cut(float equal, uint32_t up_to) : low(nextafterf(equal, __builtin_inff())), at(equal), last(up_to) {}
    template <int kVec>
    __device__ __forceinline__ void keep(uint32_t first, const float (&x)[kVec], bool (&in)[kVec]) const {
#pragma unroll
        for (int i = 0; i < kVec; ++i) in[i] = x[i] >= low;
        if (at < low) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) in[i] |= x[i] == at && first + i <= last;
        }
    }
    __device__ __forceinline__ float lowest() const { return at; }
    // Without logits below `floor`.
    __device__ __forceinline__ Cut above(float floor) const { return floor > at ? Cut(fmaxf(low, floor)) : *this; }
};

// x plus what the lanes before it hold (kShift: within their 16, by that many; then the
// last lane of the rows before).
template <int kControl, int kRows>
__device__ __forceinline__ uint64_t add_from(uint64_t x) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0u, static_cast<uint32_t>(x), kControl, kRows, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0u, static_cast<uint32_t>(x >> 32), kControl, kRows, 0xf, false);
    return x + (static_cast<uint64_t>(hi) << 32 | lo);
}
// The sum of the lanes up to this one.
__device__ __forceinline__ uint64_t wave_until(uint64_t x) {
    x = add_from<0x111, 0xf>(x);  // row_shr
    x = add_from<0x112, 0xf>(x);
    x = add_from<0x114, 0xf>(x);
    x = add_from<0x118, 0xf>(x);
    x = add_from<0x142, 0xa>(x);  // row_bcast of lane 15
    return add_from<0x143, 0xc>(x);  // and of lane 31
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
    x = wave_until(x);
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(x), 63);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(x >> 32), 63);
    return static_cast<uint64_t>(hi) << 32 | lo;
}
// The sum of the lower lanes' values.
__device__ __forceinline__ uint64_t wave_before(uint64_t x) { return wave_until(x) - x; }

// A row in units of a vector a lane, which the wavefronts take in turns, kAhead loaded
// together.  2^shift units are a batch.
template <class T, int kThreads>
struct Row {
    static constexpr int kWaves = kThreads / 64;
    static constexpr int kVec = 8, kUnit = 64 * kVec, kAhead = 4;
    const T* at;
    uint32_t vocab, units, shift = 0;

    __device__ __forceinline__ Row(const T* row, int64_t n) : at(row), vocab(static_cast<uint32_t>(n)), units((vocab + kUnit - 1) / kUnit) {
        while (units > uint32_t(kBatches) << shift) ++shift;
    }
    __device__ __forceinline__ uint32_t batches() const { return (units + (1u << shift) - 1) >> shift; }
    __device__ __forceinline__ uint32_t batch_of(uint32_t index) const { return index / kUnit >> shift; }
    __device__ __forceinline__ Pack<T, kVec> load(uint32_t first) const {
        Pack<T, kVec> v;
        if (first + kVec <= vocab) {
            v = *reinterpret_cast<const Pack<T, kVec>*>(at + first);
        } else {
#pragma unroll
            for (int i = 0; i < kVec; ++i) v.v[i] = first + i < vocab ? at[first + i] : static_cast<T>(-__builtin_inff());
        }
        return v;
    }
    static __device__ __forceinline__ void values(const Pack<T, kVec>& v, float (&x)[kVec]) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) x[i] = static_cast<float>(v.v[i]);
    }
    // f(unit, first index of the lane's values, the values; -inf behind the row).
    template <class F>
    __device__ __forceinline__ void each(F f) const {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        for (uint32_t u = wave; u < units; u += kWaves * kAhead) {
            const uint32_t first = u * kUnit + (threadIdx.x & 63) * kVec;
            Pack<T, kVec> v[kAhead];
            if ((u + (kAhead - 1) * kWaves + 1) * kUnit <= vocab) {  // whole units: the loads go out together
#pragma unroll
                for (int a = 0; a < kAhead; ++a) v[a] = *reinterpret_cast<const Pack<T, kVec>*>(at + (first + a * kWaves * kUnit));
            } else {
#pragma unroll
                for (int a = 0; a < kAhead; ++a) v[a] = load(first + a * kWaves * kUnit);
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                if (u + a * kWaves >= units) break;
                float x[kVec];
                values(v[a], x);
                f(u + a * kWaves, first + a * kWaves * kUnit, x);
            }
        }
    }
};

// The wavefronts' sums into s.waves, and the whole sum to every thread.
template <int kThreads>
__device__ __forceinline__ uint64_t total_of(Shared<kThreads>& s, uint64_t mine) {
    mine = wave_sum(mine);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.waves[threadIdx.x >> 6] = mine;
    __syncthreads();
    uint64_t sum = 0;
    for (int w = 0; w < Shared<kThreads>::kWaves; ++w) sum += s.waves[w];
    return sum;
}

// Finds the first of `count` sums (up to kBins), taken in rising order (kDown: falling), at
// which their sum reaches target: s.chosen, with what comes before in s.before and its own
// in s.value.
template <bool kDown, int kThreads>
__device__ __forceinline__ void choose(Shared<kThreads>& s, const uint64_t* sums, uint32_t count, uint64_t target) {
    constexpr uint32_t kEach = kBins / kThreads;
    const uint32_t first = threadIdx.x * kEach;
    const auto place = [&](uint32_t i) { return kDown ? count - 1 - (first + i) : first + i; };
    uint64_t mine = 0;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) mine += first + i < count ? sums[place(i)] : 0;
    uint64_t before = wave_before(mine);
    if ((threadIdx.x & 63) == 63) s.waves[threadIdx.x >> 6] = before + mine;
    __syncthreads();
    for (int w = 0; w < static_cast<int>(threadIdx.x >> 6); ++w) before += s.waves[w];
    if (before < target && before + mine >= target) {
        for (uint32_t i = 0; i < kEach && first + i < count; ++i) {
            const uint64_t x = sums[place(i)];
            if (before < target && before + x >= target) {
                s.chosen = place(i);
                s.before = before;
                s.value = x;
            }
            before += x;
        }
    }
    __syncthreads();
}

template <int kThreads>
__device__ __forceinline__ void clear_bins(Shared<kThreads>& s) {
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads) s.bins[i] = 0;
    __syncthreads();
}
template <int kThreads>
__device__ __forceinline__ void add_to_bin(Shared<kThreads>& s, uint32_t bin, uint64_t x) {
    atomicAdd(reinterpret_cast<unsigned long long*>(&s.bins[bin]), static_cast<unsigned long long>(x));
}
// Counts, which stay within the lower word.
template <int kThreads>
__device__ __forceinline__ void add_to_bin(Shared<kThreads>& s, uint32_t bin, uint32_t x) {
    atomicAdd(reinterpret_cast<uint32_t*>(&s.bins[bin]), x);
}

// The sum of the values of the threads before this one, and of all.
template <int kThreads>
__device__ __forceinline__ uint64_t before_in_list(Shared<kThreads>& s, uint64_t x, uint64_t* all) {
    uint64_t before = wave_before(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) s.waves[threadIdx.x >> 6] = before + x;
    __syncthreads();
    uint64_t sum = 0;
    for (int w = 0; w < Shared<kThreads>::kWaves; ++w) {
        if (w == static_cast<int>(threadIdx.x >> 6)) before += sum;
        sum += s.waves[w];
    }
    *all = sum;
    return before;
}

// s.batches = the sums of `sum` (of a vector, with its terms) over the row's batches.
template <class T, int kThreads, class Sum>
__device__ __forceinline__ void add_batches(Shared<kThreads>& s, const Row<T, kThreads>& row, Sum sum) {
    constexpr int kVec = Row<T, kThreads>::kVec;
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < row.batches(); b += kThreads) s.batches[b] = 0;
    __syncthreads();
    row.each([&](uint32_t unit, uint32_t first, const float(&x)[kVec]) {
        uint64_t terms[kVec];
        const uint64_t all = wave_sum(sum(first, x, terms));
        if (all > 0 && (threadIdx.x & 63) == 0)
            atomicAdd(reinterpret_cast<unsigned long long*>(&s.batches[unit >> row.shift]), static_cast<unsigned long long>(all));
    });
    __syncthreads();
}
template <class T, int kThreads>
__device__ __forceinline__ uint64_t sum_batches(Shared<kThreads>& s, const Row<T, kThreads>& row) {
    uint64_t mine = 0;
    for (uint32_t b = threadIdx.x; b < row.batches(); b += kThreads) mine += s.batches[b];
    return total_of(s, mine);
}
// Calls found(index, logit) for the first index at which the running sum of sum's terms
// exceeds target, which is below s.batches' sum.  A wavefront a unit of its batch.
template <class T, int kThreads, class Sum, class Found>
__device__ __forceinline__ void pick(Shared<kThreads>& s, const Row<T, kThreads>& row, uint64_t target, Sum sum, Found found) {
    constexpr int kVec = Row<T, kThreads>::kVec;
    static_assert(Row<T, kThreads>::kWaves >= 2, "a batch of a vocabulary of 2^22 has two units at most");
    __syncthreads();
    choose<false>(s, s.batches, row.batches(), target + 1);
    const uint32_t wave = threadIdx.x >> 6, unit = (s.chosen << row.shift) + wave;
    const uint32_t first = unit * Row<T, kThreads>::kUnit + (threadIdx.x & 63) * kVec;
    float x[kVec];
    uint64_t terms[kVec], own = 0, all, before = s.before;
    if (wave < 1u << row.shift) {
        row.values(row.load(first), x);
        own = sum(first, x, terms);
    }
    before += before_in_list(s, own, &all);
    if (before <= target && target < before + own) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            if (before <= target && target < before + terms[i]) found(first + i, x[i]);
            before += terms[i];
        }
    }
}

// Narrows `cut` to the shortest prefix whose measure (a token's, by its logit) reaches
// target, which is above 0 and at most the kept tokens' own, by histograms over the
// logits' keys.
template <class T, int kThreads, class Measure>
__device__ __forceinline__ void narrow(Shared<kThreads>& s, const Row<T, kThreads>& row, Cut& cut, float most, uint64_t target, Measure measure) {
    constexpr int kVec = Row<T, kThreads>::kVec;
    uint32_t lo = key_of(cut.lowest()), hi = key_of(most);
    uint64_t held = 0;  // of the last bin
    for (;;) {
        const uint32_t span = hi - lo;
        const int bits = span ? 32 - __clz(span) : 0, shift = bits > kKeyBits ? bits - kKeyBits : 0;
        clear_bins(s);
        row.each([&](uint32_t, uint32_t first, const float(&x)[kVec]) {
            bool in[kVec];
            cut.keep(first, x, in);
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (in[i]) {
                    const uint32_t key = key_of(x[i]);
                    if (key >= lo && key <= hi) add_to_bin(s, (key - lo) >> shift, measure(x[i]));
                }
        });
        __syncthreads();
        choose<true>(s, s.bins, kBins, target);
        target -= s.before;
        held = s.value;
        lo += s.chosen << shift;
        if (shift == 0) break;
        const uint32_t end = lo + ((1u << shift) - 1);
        hi = end < hi ? end : hi;
    }
    // of the tokens at the cut, the first `wanted`
    const float at = logit_of(lo);
    const uint64_t each = measure(at), wanted = (target + each - 1) / each;
    const bool some = wanted * each < held;
    const Cut old = cut;
    cut = at == old.at && at < old.low ? old : Cut(at);
    if (!some) return;
    const auto ties = [&](uint32_t first, const float(&x)[kVec], uint64_t(&n)[kVec]) {
        bool in[kVec];
        old.keep(first, x, in);
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            n[i] = x[i] == at && in[i] ? 1 : 0;
            sum += n[i];
        }
        return sum;
    };
    add_batches(s, row, ties);
    pick(s, row, wanted - 1, ties, [&](uint32_t index, float) { s.chosen = index; });
    __syncthreads();
    cut = Cut(at, s.chosen);
}

// List entries: in the order of logits, and in that of indices.
__device__ __forceinline__ uint64_t entry(float x, uint32_t index) {
    return static_cast<uint64_t>(~key_of(x)) << 32 | index;
}
__device__ __forceinline__ float logit_of_entry(uint64_t e) { return logit_of(~static_cast<uint32_t>(e >> 32)); }
__device__ __forceinline__ uint64_t turned(uint64_t e) { return e << 32 | e >> 32; }
constexpr uint64_t kNoEntry = ~uint64_t(0);

// The value of another lane by the data path between lanes; every lane takes part.
template <int kControl>
__device__ __forceinline__ uint64_t from_lane(uint64_t x) {
    const uint32_t lo = __builtin_amdgcn_update_dpp(0u, static_cast<uint32_t>(x), kControl, 0xf, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0u, static_cast<uint32_t>(x >> 32), kControl, 0xf, 0xf, false);
    return static_cast<uint64_t>(hi) << 32 | lo;
}
// The value of the lane whose number differs in bit j: where a lane's neighbours reach it,
// without shared memory.
template <uint32_t j>
__device__ __forceinline__ uint64_t across(uint64_t x) {
    if constexpr (j == 1)
        return from_lane<0xb1>(x);  // of its quad
    else if constexpr (j == 2)
        return from_lane<0x4e>(x);
    else if constexpr (j == 8)
        return from_lane<0x128>(x);  // eight on, around its sixteen
    else
        return __shfl_xor(x, j);
}
// A wavefront's entries, rising by lane; k: runs of k / 2 that are sorted, up and down in
// turns.  Each distance is a constant, so that a step is a few instructions: a row of 50257
// float32 logits with top_k 50 in 14.1 us, in a loop over the distances 16.5.
template <uint32_t k = 2, uint32_t j = k / 2>
__device__ __forceinline__ uint64_t sorted_lanes(uint64_t mine) {
    const uint32_t t = threadIdx.x & 63;
    const uint64_t other = across<j>(mine);
    const bool lower = ((t & j) == 0) == ((t & k) == 0);
    mine = (mine < other) == lower ? mine : other;
    if constexpr (j > 1)
        return sorted_lanes<k, j / 2>(mine);
    else if constexpr (k < 64)
        return sorted_lanes<k * 2>(mine);
    else
        return mine;
}

// Sorts the threads' entries, of the first n threads, rising; kNoEntry behind them.  Up to
// 64 stay within a wavefront.
template <int kThreads>
__device__ __forceinline__ uint64_t sorted(Shared<kThreads>& s, uint32_t n, uint64_t mine) {
    const uint32_t t = threadIdx.x;
    uint32_t size = 64;
    while (size < n) size *= 2;
    if (size == 64) return t < 64 ? sorted_lanes(mine) : kNoEntry;
    for (uint32_t k = 2; k <= size; k *= 2)
        for (uint32_t j = k / 2; j > 0; j /= 2) {
            uint64_t other;
            if (j >= 64) {
                __syncthreads();
                s.list[t] = mine;
                __syncthreads();
                other = s.list[t ^ j];
            } else {
                other = __shfl_xor(mine, j);
            }
            const bool lower = ((t & j) == 0) == ((t & k) == 0);
            mine = (mine < other) == lower ? mine : other;
        }
    return mine;
}

// Adds the logits of a vector for which `in` holds to the list, in no particular order;
// s.count counts them, of which kList at most are listed.
template <int kThreads, int kVec>
__device__ __forceinline__ void enlist(Shared<kThreads>& s, uint32_t first, const float (&x)[kVec], const bool (&in)[kVec]) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < kVec; ++i) any |= in[i];
    if (__ballot(any) == 0) return;
#pragma unroll
    for (int i = 0; i < kVec; ++i)
        if (in[i]) {
            const uint32_t at = atomicAdd(&s.count, 1u);
            if (at < Shared<kThreads>::kList) s.list[at] = entry(x[i], first + i);
        }
}

// Bound by vector arithmetic, 25 instructions for each weight: 2048 rows of 50257 bfloat16
// logits in 138 to 148 us, with top_p 0.95 269, with top_k 50 98 and with T = 0, two
// readings alone, 79 (5.2 TB/s); one binary32 row in 21, 41, 13.4 and 7 us.  (Logits from
// memory; of one batch drawn from again and again, which the last cache holds in part,
// 129, 261, 85 and 68.)
template <class T, int kThreads>
__global__ __launch_bounds__(kThreads, 4) void sample_kernel(SampleCall call, int bits) {
    constexpr int kList = kThreads, kListK = kThreads / 2, kVec = Row<T, kThreads>::kVec;
    __shared__ Shared<kThreads> s;
    const int64_t r = blockIdx.x;
    if (threadIdx.x < kExpSteps) s.powers[threadIdx.x] = exp2(threadIdx.x / static_cast<double>(kExpSteps));
    Row<T, kThreads> row(static_cast<const T*>(call.logits.at) + r * call.logits.stride, call.vocab);
    const micro_sampling& set = call.sampling;
    const double t = set.temperatures ? static_cast<double>(set.temperatures[r]) : set.temperature;
    const double p = set.top_ps ? static_cast<double>(set.top_ps[r]) : set.top_p;
    const double least = set.min_ps ? static_cast<double>(set.min_ps[r]) : set.min_p;
    const int64_t k = set.top_ks ? set.top_ks[r] : set.top_k;

    // the threads' largest logits, and the row's
    float top = -__builtin_inff();
    row.each([&](uint32_t, uint32_t, const float(&x)[kVec]) {
#pragma unroll
        for (int i = 0; i < kVec; ++i) top = fmaxf(top, x[i]);
    });
    float most = top;
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    if ((threadIdx.x & 63) == 0) s.waves[threadIdx.x >> 6] = __float_as_uint(most);
    __syncthreads();
    for (int w = 0; w < Shared<kThreads>::kWaves; ++w) most = fmaxf(most, __uint_as_float(static_cast<uint32_t>(s.waves[w])));
    const auto answer = [&](int64_t id, float logprob) {
        if (call.ids.wide)
            static_cast<int64_t*>(const_cast<void*>(call.ids.at))[r] = id;
        else
            static_cast<int32_t*>(const_cast<void*>(call.ids.at))[r] = static_cast<int32_t>(id);
        if (call.logprobs) call.logprobs[r] = logprob;
    };
    if (!(most > -__builtin_inff())) {
        if (threadIdx.x == 0) answer(-1, __builtin_nanf(""));
        return;
    }
    if (!(t > 0.0)) {
        if (threadIdx.x == 0) s.chosen = 0xffffffffu;
        __syncthreads();
        uint32_t index = 0xffffffffu;
        row.each([&](uint32_t, uint32_t first, const float(&x)[kVec]) {
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (x[i] == most && first + i < index) index = first + i;
        });
        if (index != 0xffffffffu) atomicMin(&s.chosen, index);
        __syncthreads();
        if (threadIdx.x == 0) answer(s.chosen, 0.0f);
        return;
    }
    const float u = call.uniforms[r];
    const auto target_of = [&](uint64_t total) {
        return u > 0.0f ? u < 1.0f ? share_of(u, total, false) : total - 1 : 0;
    };
    const auto prefix_of = [&](uint64_t total) {
        const uint64_t wanted = p < 1.0 ? share_of(p, total, true) : p >= 1.0 || p != p ? total : 0;
        return wanted > 0 ? wanted : 1;
    };
    if (most == __builtin_inff()) {  // equal weights of the infinite logits, of 1 each
        const auto infinite = [&](uint32_t, const float(&x)[kVec], uint64_t(&n)[kVec]) {
            uint64_t sum = 0;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                n[i] = x[i] == most ? 1 : 0;
                sum += n[i];
            }
            return sum;
        };
        add_batches(s, row, infinite);
        uint64_t kept = sum_batches(s, row);
        if (k > 0 && static_cast<uint64_t>(k) < kept) kept = static_cast<uint64_t>(k);
        kept = (prefix_of(kept << bits) + (uint64_t(1) << bits) - 1) >> bits;
        pick(s, row, target_of(kept << bits) >> bits, infinite,
             [&](uint32_t index, float) { answer(index, static_cast<float>(-log(static_cast<double>(kept)))); });
        return;
    }

    constexpr double kLn2 = 0.6931471805599453;
    const double warm = fmax(t, 1e-300);
    // logits below weigh nothing (rounded down: of the next lower binary32)
    const double range = (bits + 2) * kLn2 * warm;
    const float floor = fmaxf(nextafterf(static_cast<float>(static_cast<double>(most) - range), -__builtin_inff()), kLowest);
    const Weigher weigher{s.powers, static_cast<double>(most), kExpSteps / kLn2 / warm, -(bits + 2.0) * kExpSteps, bits << 20};
    const auto weigh = [&](float x) { return weigher.weight(x); };
    // the smallest logit that min_p keeps, by its key (the exponent rises with the logit)
    float limit = kLowest;
    if (least > 0.0) {
        const double lowest = log(least);
        uint32_t below = key_of(kLowest) - 1, kept = key_of(most);
        while (kept - below > 1) {
            const uint32_t middle = below + (kept - below) / 2;
            if (weigher.exponent(logit_of(middle)) < lowest)
                below = middle;
            else
                kept = middle;
        }
        limit = logit_of(kept);
    }
    const auto finish = [&](float x, uint32_t index, uint64_t total) {
        const double share = static_cast<double>(total) * __builtin_bit_cast(double, static_cast<uint64_t>(1023 - bits) << 52);
        answer(index, static_cast<float>(weigher.exponent(x) - log(share)));
    };
    Cut cut(kLowest);

    if (k > 0 && k <= kListK) {
        // a lower bound of the k-th logit: k threads' maxima reach it
        clear_bins(s);
        float bottom = top > -__builtin_inff() ? top : most;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) bottom = fminf(bottom, __shfl_xor(bottom, d));
        if ((threadIdx.x & 63) == 0) s.waves[threadIdx.x >> 6] = __float_as_uint(bottom);
        __syncthreads();
        for (int w = 0; w < Shared<kThreads>::kWaves; ++w) bottom = fminf(bottom, __uint_as_float(static_cast<uint32_t>(s.waves[w])));
        const uint32_t lo = key_of(bottom), span = key_of(most) - lo;
        const int width = span ? 32 - __clz(span) : 0, shift = width > kKeyBits ? width - kKeyBits : 0;
        if (top > -__builtin_inff()) add_to_bin(s, (key_of(top) - lo) >> shift, 1u);
        if (threadIdx.x == 0) {
            add_to_bin(s, 0, static_cast<uint32_t>(kListK));  // the lowest bin holds as many as are wanted
            s.count = 0;
        }
        __syncthreads();
        choose<true>(s, s.bins, kBins, static_cast<uint64_t>(k));
        const float bound = s.chosen > 0 ? logit_of(lo + (s.chosen << shift)) : kLowest;
        row.each([&](uint32_t, uint32_t first, const float(&x)[kVec]) {
            bool in[kVec];
#pragma unroll
            for (int i = 0; i < kVec; ++i) in[i] = x[i] >= bound;
            enlist(s, first, x, in);
        });
        __syncthreads();
        const uint32_t n = s.count;
        if (n <= kList) {
            uint64_t mine = threadIdx.x < n ? s.list[threadIdx.x] : kNoEntry;
            mine = sorted(s, n, mine);
            const uint32_t first = n < static_cast<uint64_t>(k) ? n : static_cast<uint32_t>(k);
            const auto weight_of = [&](bool kept, float x) { return kept ? weigh(x) : 0; };
            uint64_t total;
            float x = logit_of_entry(mine);
            const uint64_t before = before_in_list(s, weight_of(threadIdx.x < first, x), &total);
            const bool kept = threadIdx.x < first && before < prefix_of(total) && x >= limit;
            mine = sorted(s, first, kept ? turned(mine) : kNoEntry);
            const bool there = mine != kNoEntry;
            x = logit_of_entry(turned(mine));
            const uint64_t w = weight_of(there, x), lower = before_in_list(s, w, &total), target = target_of(total);
            if (lower <= target && target < lower + w) finish(x, static_cast<uint32_t>(turned(mine)), total);
            return;
        }
    }
    if (k > 0) {
        uint64_t live = 0;
        row.each([&](uint32_t, uint32_t, const float(&x)[kVec]) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) live += x[i] >= kLowest ? 1 : 0;
        });
        live = total_of(s, live);
        if (static_cast<uint64_t>(k) < live)
            narrow(s, row, cut, most, static_cast<uint64_t>(k), [](float) { return uint32_t(1); });
    }

    // The weights of a vector's logits that `in` takes and their sum: side by side, without a
    // branch around each, and not at all where the wavefront takes none.
    const auto weigh_all = [&](const float(&x)[kVec], const bool(&in)[kVec], uint64_t(&w)[kVec]) {
        bool any = false;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            any |= in[i];
            w[i] = 0;
        }
        uint64_t sum = 0;
        if (__ballot(any) == 0) return sum;
#pragma unroll
        for (int i = 0; i < kVec; ++i) {
            const uint64_t biased = weigher.biased(in[i] ? x[i] : -__builtin_inff());  // which weighs 0
            w[i] = biased - Weigher::kBias;
            sum += biased;
        }
        return sum - kVec * Weigher::kBias;
    };
    bool summed = false;  // s.batches hold what is kept
    if (p < 1.0) {
        // weights by equal steps down from the largest logit; a larger step never holds
        // larger logits, since subtraction and multiplication keep their order
        const float per = static_cast<float>(kBins / range);
        const auto bin_of = [&](float x) {
            const float b = (most - x) * per;
            return b < kBins - 1 ? static_cast<uint32_t>(b) : kBins - 1u;
        };
        const Cut weighing = cut.above(floor);
        if (threadIdx.x == 0) s.count = 0;
        clear_bins(s);
        row.each([&](uint32_t, uint32_t first, const float(&x)[kVec]) {
            bool in[kVec];
            uint64_t w[kVec];
            weighing.keep(first, x, in);
            (void)weigh_all(x, in, w);
#pragma unroll
            for (int i = 0; i < kVec; ++i)
                if (w[i] > 0) add_to_bin(s, bin_of(x[i]), w[i]);
        });
        __syncthreads();
        uint64_t mine = 0;
#pragma unroll
        for (int i = 0; i < kBins / kThreads; ++i) mine += s.bins[threadIdx.x + i * kThreads];
        const uint64_t wanted = prefix_of(total_of(s, mine));
        __syncthreads();
        choose<false>(s, s.bins, kBins, wanted);
        // the batches' sums of what the bins above hold, and the list of the cut's own
        const uint32_t chosen = s.chosen;
        const uint64_t above = s.before;
        add_batches(s, row, [&](uint32_t first, const float(&x)[kVec], uint64_t(&w)[kVec]) {
            bool in[kVec], here[kVec];
            weighing.keep(first, x, in);
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const uint32_t b = bin_of(x[i]);
                here[i] = in[i] && b == chosen;
                in[i] = in[i] && b < chosen;
            }
            enlist(s, first, x, here);
            return weigh_all(x, in, w);
        });
        const uint32_t n = s.count;
        if (n <= kList) {
            const uint64_t e = sorted(s, n, threadIdx.x < n ? s.list[threadIdx.x] : kNoEntry);
            uint64_t all;
            const uint64_t w = e != kNoEntry ? weigh(logit_of_entry(e)) : 0;
            const uint64_t before = above + before_in_list(s, w, &all);
            if (before < wanted && w > 0) {
                if (before + w >= wanted) s.value = e;
                atomicAdd(reinterpret_cast<unsigned long long*>(&s.batches[row.batch_of(static_cast<uint32_t>(e))]),
                          static_cast<unsigned long long>(w));
            }
            __syncthreads();
            cut = Cut(logit_of_entry(s.value), static_cast<uint32_t>(s.value));
            summed = !(cut.at < limit);
        } else {
            narrow(s, row, cut, most, wanted, weigh);
        }
    }
    cut = cut.above(fmaxf(floor, limit));
    const auto weights_of = [&](uint32_t first, const float(&x)[kVec], uint64_t(&w)[kVec]) {
        bool in[kVec];
        cut.keep(first, x, in);
        return weigh_all(x, in, w);
    };
    if (!summed) add_batches(s, row, weights_of);
    const uint64_t total = sum_batches(s, row);
    pick(s, row, target_of(total), weights_of, [&](uint32_t index, float x) { finish(x, index, total); });
}

}  // namespace

template <class T>
hipError_t launch_rows(const SampleCall& call, hipStream_t stream) {
    const int bits = weight_bits(call.vocab);
    const dim3 grid(static_cast<uint32_t>(call.rows));
    // Rows for every compute unit: two workgroups each, one at work while the other waits
    // (2048 rows of 50257 bfloat16 logits, top_p 0.95, in 269 us for 379; 300 rows in 76
    // for 92), unless a top_k for all needs the larger workgroup's list (top_k 500 in 264
    // us for 380; one a row, which the host does not see, takes the 380).
    const bool longer = !call.sampling.top_ks && call.sampling.top_k > 256 && call.sampling.top_k <= 512;
    if (call.rows > call.compute_units && !longer) return launch(sample_kernel<T, 512>, grid, 512, stream, call, bits);
    return launch(sample_kernel<T, 1024>, grid, 1024, stream, call, bits);
}

hipError_t launch_sample(const SampleCall& call, hipStream_t stream) {
    if (call.rows == 0) return hipSuccess;
    switch (call.logits.type) {
        case MICRO_TYPE_F32: return launch_rows<float>(call, stream);
        case MICRO_TYPE_F16: return launch_rows<f16>(call, stream);
        default: return launch_rows<bf16>(call, stream);
    }
}

}  // namespace micro

// gfx950 kernel that draws a token from each row of logits:
//   m = max l,   w_i = exp((l_i - m) / T),   ordered by (logit descending, index)
//   kept: the first top_k, of those the shortest prefix that reaches top_p of
//   their weight, of those w_i >= min_p
//   token: the first index where the running sum of kept weights exceeds u times
//   their sum
// Weights are computed in binary64 and rounded to whole multiples of 2^-f; their
// sums are of 64-bit integers and exact, so the token does not depend on how a row
// is divided, and a border between two tokens lies where binary64 sums have it
// to 2^-f.  The two cuts along the order are found without sorting, by histograms
// over the logits' bits: each level spreads the interval that holds the cut over
// kBins bins of counts (top_k) or weights (top_p).
#include "sample_kernel.h"

#include "launch.h"
#include "value_types.h"

namespace micro {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBinBits = 11, kBins = 1 << kBinBits;
constexpr int kExpSteps = 64;  // of the table of 2^(j / 64)

// Bits of a logit in its order: larger logits have larger keys, equal ones (-0
// and 0) the same; 0 where it has no part (-inf, NaN).
template <class T>
__device__ __forceinline__ uint32_t key_of(T x) {
    if constexpr (sizeof(T) == 4) {
        const uint32_t u = __float_as_uint(x + 0.0f);
        return x > -__builtin_inff() ? u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u) : 0u;
    } else {
        const uint16_t u = __builtin_bit_cast(uint16_t, x);
        const uint32_t v = u == 0x8000u ? 0u : u;
        return static_cast<float>(x) > -__builtin_inff() ? v ^ ((v >> 15) ? 0xffffu : 0x8000u) : 0u;
    }
}
template <class T>
__device__ __forceinline__ float logit_of(uint32_t key) {
    if constexpr (sizeof(T) == 4) {
        return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu));
    } else {
        const uint16_t u = static_cast<uint16_t>(key ^ ((key >> 15) ? 0x8000u : 0xffffu));
        return static_cast<float>(__builtin_bit_cast(T, u));
    }
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

struct Settings {
    double inverse;  // 1 / temperature
    double p, least;  // least: the smallest (l - m) / T that min_p keeps
    int64_t k;
};

struct Shared {
    double powers[kExpSteps];
    uint64_t bins[kBins];
    uint64_t waves[kWaves];
    uint64_t value;   // one thread's answer to all
    uint64_t before;
    uint32_t chosen;
};

// Weights of one row.
struct Weigher {
    const double* powers;
    double most, inverse;
    int bits;

    // exp(y) 2^bits to the nearest integer, y <= 0, by a table of 2^(j/64) and the
    // series of exp to the fifth power over the rest, which is below 2^-7.5 (Tang's
    // method, 1989); the series ends at 3.5e-17.
    __device__ __forceinline__ uint64_t weight(double y) const {
        y = __builtin_fmax(y, -100.0);  // less than 2^-144; NaN (an infinite rest) too
        const double n = __builtin_rint(y * (kExpSteps * 1.4426950408889634));
        const double r = __builtin_fma(n, -0.6931471805599453 / kExpSteps, y);
        const int i = static_cast<int>(n);
        double s = __builtin_fma(r, 1.0 / 120, 1.0 / 24);
        s = __builtin_fma(r, s, 1.0 / 6);
        s = __builtin_fma(r, s, 0.5);
        s = __builtin_fma(r, s, 1.0);
        s = __builtin_fma(r, s, 1.0);
        const double unit = __builtin_bit_cast(double, static_cast<uint64_t>(1023 + (i >> 6) + bits) << 52);
        // adding 2^52 leaves the integer in the last bits
        const double sum = __builtin_fma(s * powers[i & (kExpSteps - 1)], unit, 4503599627370496.0);
        return __builtin_bit_cast(uint64_t, sum) & ((uint64_t(1) << 52) - 1);
    }
    __device__ __forceinline__ double exponent(float logit) const {
        const double x = logit;
        return x == most ? 0.0 : (x - most) * inverse;
    }
};

// The kept prefix of the order: logits above `key`, and equal ones up to index
// `last`.
struct Cut {
    uint32_t key, last;
    __device__ bool keeps(uint32_t k, uint32_t index) const { return k > key || (k == key && index <= last); }
};

__device__ __forceinline__ uint64_t wave_sum(uint64_t x) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
// The sum of the lower lanes' values.
__device__ __forceinline__ uint64_t wave_before(uint64_t x) {
    uint64_t sum = x;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t other = __shfl_up(sum, d);
        sum += lane >= d ? other : 0;
    }
    return sum - x;
}

// A row, divided among the wavefronts into runs of indices.
template <class T>
struct Row {
    static constexpr int kVec = 16 / sizeof(T), kStep = 64 * kVec;
    const T* at;
    uint32_t vocab, run;  // values, and those of a wavefront

    __device__ Row(const T* row, int64_t n) : at(row), vocab(static_cast<uint32_t>(n)) {
        run = (vocab + kWaves * kStep - 1) / (kWaves * kStep) * kStep;
    }
    // f(first index of the lane's values, their keys; 0 behind the row), step by
    // step over the run of a wavefront, while f returns true.
    template <class F>
    __device__ __forceinline__ void each(int wave, F f) const {
        const uint32_t begin = wave * run, end = begin + run < vocab ? begin + run : vocab;
        for (uint32_t base = begin; base < end; base += kStep) {
            const uint32_t first = base + (threadIdx.x & 63) * kVec;
            uint32_t keys[kVec];
            if (first + kVec <= vocab) {
                const Pack<T, kVec> v = *reinterpret_cast<const Pack<T, kVec>*>(at + first);
#pragma unroll
                for (int i = 0; i < kVec; ++i) keys[i] = key_of<T>(v.v[i]);
            } else {
#pragma unroll
                for (int i = 0; i < kVec; ++i) keys[i] = first + i < vocab ? key_of<T>(at[first + i]) : 0u;
            }
            if (!f(first, keys)) return;
        }
    }
};

// The wavefronts' values, and their sum to every thread.
__device__ __forceinline__ uint64_t total_of(Shared& s, uint64_t mine) {
    mine = wave_sum(mine);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.waves[threadIdx.x >> 6] = mine;
    __syncthreads();
    uint64_t sum = 0;
    for (int w = 0; w < kWaves; ++w) sum += s.waves[w];
    return sum;
}

// The wavefront in which the sum of s.waves passes `target`, and what comes before.
__device__ __forceinline__ int wave_at(const Shared& s, uint64_t target, uint64_t* before) {
    uint64_t sum = 0;
    for (int w = 0; w < kWaves - 1; ++w) {
        if (sum + s.waves[w] > target) {
            *before = sum;
            return w;
        }
        sum += s.waves[w];
    }
    *before = sum;
    return kWaves - 1;
}

// Narrows `cut` to the shortest prefix whose measure (a token's, by its key)
// reaches target, which is above 0 and at most the kept tokens' own.
template <class T, class Measure>
__device__ void narrow(Shared& s, const Row<T>& row, Cut& cut, uint32_t most, uint64_t target, Measure measure) {
    uint32_t lo = cut.key, hi = most;
    uint64_t held = 0;  // of the last bin
    for (;;) {
        const uint32_t span = hi - lo;
        const int bits = span ? 32 - __clz(span) : 0, shift = bits > kBinBits ? bits - kBinBits : 0;
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kThreads) s.bins[i] = 0;
        __syncthreads();
        row.each(threadIdx.x >> 6, [&](uint32_t first, const uint32_t(&keys)[Row<T>::kVec]) {
#pragma unroll
            for (int i = 0; i < Row<T>::kVec; ++i)
                if (keys[i] >= lo && keys[i] <= hi && cut.keeps(keys[i], first + i))
                    atomicAdd(reinterpret_cast<unsigned long long*>(&s.bins[(keys[i] - lo) >> shift]),
                              static_cast<unsigned long long>(measure(keys[i])));
            return true;
        });
        __syncthreads();
        // from the top bin down, kBins / kThreads a thread
        constexpr int kEach = kBins / kThreads;
        const int top = kBins - 1 - static_cast<int>(threadIdx.x) * kEach;
        uint64_t mine = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) mine += s.bins[top - i];
        uint64_t before = wave_before(mine);
        if ((threadIdx.x & 63) == 63) s.waves[threadIdx.x >> 6] = before + mine;
        __syncthreads();
        for (int w = 0; w < static_cast<int>(threadIdx.x >> 6); ++w) before += s.waves[w];
        if (before < target && before + mine >= target) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const uint64_t x = s.bins[top - i];
                if (before < target && before + x >= target) {
                    s.chosen = top - i;
                    s.before = before;
                    s.value = x;
                }
                before += x;
            }
        }
        __syncthreads();
        target -= s.before;
        held = s.value;
        lo += s.chosen << shift;
        if (shift == 0) break;
        const uint32_t end = lo + ((1u << shift) - 1);
        hi = end < hi ? end : hi;
    }
    // of the tokens at the cut, the first `wanted`
    const uint64_t each = measure(lo), wanted = (target + each - 1) / each;
    const bool some = wanted * each < held;
    const Cut old = cut;
    cut = {lo, lo == old.key ? old.last : 0xffffffffu};
    if (!some) return;
    const auto count = [&](uint32_t first, const uint32_t(&keys)[Row<T>::kVec]) {
        uint64_t n = 0;
#pragma unroll
        for (int i = 0; i < Row<T>::kVec; ++i) n += keys[i] == lo && old.keeps(keys[i], first + i) ? 1 : 0;
        return n;
    };
    uint64_t mine = 0;
    row.each(threadIdx.x >> 6, [&](uint32_t first, const uint32_t(&keys)[Row<T>::kVec]) {
        mine += count(first, keys);
        return true;
    });
    (void)total_of(s, mine);
    uint64_t before;
    const int wave = wave_at(s, wanted - 1, &before);
    if (static_cast<int>(threadIdx.x >> 6) == wave) {
        row.each(wave, [&](uint32_t first, const uint32_t(&keys)[Row<T>::kVec]) {
            const uint64_t n = count(first, keys), lower = before + wave_before(n);
            if (lower < wanted && lower + n >= wanted) {
                uint64_t left = wanted - lower;
#pragma unroll
                for (int i = 0; i < Row<T>::kVec; ++i)
                    if (keys[i] == lo && old.keeps(keys[i], first + i) && --left == 0) s.chosen = first + i;
            }
            before += wave_sum(n);
            return before < wanted;
        });
    }
    __syncthreads();
    cut.last = s.chosen;
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleCall call, int bits) {
    __shared__ Shared s;
    const int64_t r = blockIdx.x;
    if (threadIdx.x < kExpSteps) s.powers[threadIdx.x] = exp2(threadIdx.x / static_cast<double>(kExpSteps));
    const Row<T> row(static_cast<const T*>(call.logits.at) + r * call.logits.stride, call.vocab);
    const micro_sampling& set = call.sampling;
    const double t = set.temperatures ? static_cast<double>(set.temperatures[r]) : set.temperature;
    const double p = set.top_ps ? static_cast<double>(set.top_ps[r]) : set.top_p;
    const double least = set.min_ps ? static_cast<double>(set.min_ps[r]) : set.min_p;
    const int64_t k = set.top_ks ? set.top_ks[r] : set.top_k;

    // the largest logit, the first of its index, and how many have a part
    uint64_t best = 0, live = 0;
    row.each(threadIdx.x >> 6, [&](uint32_t first, const uint32_t(&keys)[Row<T>::kVec]) {
#pragma unroll
        for (int i = 0; i < Row<T>::kVec; ++i) {
            const uint64_t x = static_cast<uint64_t>(keys[i]) << 32 | (0xffffffffu - (first + i));
            if (keys[i]) {
                best = x > best ? x : best;
                ++live;
            }
        }
        return true;
    });
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const uint64_t x = __shfl_xor(best, d);
        best = x > best ? x : best;
    }
    if ((threadIdx.x & 63) == 0) s.bins[threadIdx.x >> 6] = best;
    live = total_of(s, live);
    for (int w = 0; w < kWaves; ++w) best = s.bins[w] > best ? s.bins[w] : best;
    const uint32_t most = static_cast<uint32_t>(best >> 32);
    const auto answer = [&](int64_t id, float logprob) {
        if (call.ids.wide)
            static_cast<int64_t*>(const_cast<void*>(call.ids.at))[r] = id;
        else
            static_cast<int32_t*>(const_cast<void*>(call.ids.at))[r] = static_cast<int32_t>(id);
        if (call.logprobs) call.logprobs[r] = logprob;
    };
    if (live == 0 || !(t > 0.0)) {
        if (threadIdx.x == 0) {
            if (live == 0)
                answer(-1, __builtin_nanf(""));
            else
                answer(0xffffffffu - static_cast<uint32_t>(best), 0.0f);
        }
        return;
    }

    const Weigher weigher{s.powers, static_cast<double>(logit_of<T>(most)), 1.0 / t, bits};
    Cut cut{1, 0xffffffffu};
    if (k > 0 && static_cast<uint64_t>(k) < live)
        narrow<T>(s, row, cut, most, static_cast<uint64_t>(k), [](uint32_t) { return uint64_t(1); });
    const auto weigh = [&](uint32_t key) { return weigher.weight(weigher.exponent(logit_of<T>(key))); };
    const auto sum = [&](double at_least) {
        uint64_t mine = 0;
        row.each(threadIdx.x >> 6, [&](uint32_t first, const uint32_t(&keys)[Row<T>::kVec]) {
#pragma unroll
            for (int i = 0; i < Row<T>::kVec; ++i)
                if (keys[i] && cut.keeps(keys[i], first + i)) {
                    const double y = weigher.exponent(logit_of<T>(keys[i]));
                    if (!(y < at_least)) mine += weigher.weight(y);
                }
            return true;
        });
        return total_of(s, mine);
    };
    const double lowest = least > 0.0 ? log(least) : -__builtin_inf();
    uint64_t total = sum(p < 1.0 ? -__builtin_inf() : lowest);
    if (p < 1.0) {
        const uint64_t wanted = share_of(p, total, true);
        narrow<T>(s, row, cut, most, wanted > 0 ? wanted : 1, weigh);
        total = sum(lowest);
    }
    const float u = call.uniforms[r];
    const uint64_t target = u > 0.0f ? u < 1.0f ? share_of(u, total, false) : total - 1 : 0;
    uint64_t before;
    const int wave = wave_at(s, target, &before);
    if (static_cast<int>(threadIdx.x >> 6) != wave) return;
    row.each(wave, [&](uint32_t first, const uint32_t(&keys)[Row<T>::kVec]) {
        uint64_t w[Row<T>::kVec], mine = 0;
#pragma unroll
        for (int i = 0; i < Row<T>::kVec; ++i) {
            w[i] = 0;
            if (keys[i] && cut.keeps(keys[i], first + i)) {
                const double y = weigher.exponent(logit_of<T>(keys[i]));
                if (!(y < lowest)) w[i] = weigher.weight(y);
            }
            mine += w[i];
        }
        uint64_t lower = before + wave_before(mine);
        if (lower <= target && target < lower + mine) {
#pragma unroll
            for (int i = 0; i < Row<T>::kVec; ++i) {
                if (lower <= target && target < lower + w[i])
                    answer(first + i, static_cast<float>(weigher.exponent(logit_of<T>(keys[i])) -
                                                         log(static_cast<double>(total) *
                                                             __builtin_bit_cast(double, static_cast<uint64_t>(1023 - bits) << 52))));
                lower += w[i];
            }
        }
        before += wave_sum(mine);
        return before <= target;
    });
}

}  // namespace

hipError_t launch_sample(const SampleCall& call, hipStream_t stream) {
    if (call.rows == 0) return hipSuccess;
    const int bits = weight_bits(call.vocab);
    const dim3 grid(static_cast<uint32_t>(call.rows));
    switch (call.logits.type) {
        case MICRO_TYPE_F32: return launch(sample_kernel<float>, grid, kThreads, stream, call, bits);
        case MICRO_TYPE_F16: return launch(sample_kernel<f16>, grid, kThreads, stream, call, bits);
        default: return launch(sample_kernel<bf16>, grid, kThreads, stream, call, bits);
    }
}

}  // namespace micro

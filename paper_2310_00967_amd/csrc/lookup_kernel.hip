// gfx950 kernels of the token table: the lookup of rows with scaling, and its
// gradient by sorted tokens.
//   lookup    out[t] = scale * table[ids[t]]: a gather, bound by HBM (16384 rows
//             of 4 KB in 16 to 17 us, 5.2 TB/s).
//   gradient  table[v] (+)= scale * sum of grad[t] over the tokens with id v.
// The gradient's tokens are sorted by id (stably, so a row's terms keep their
// order and the binary32 sum is the same on every run) and cut into chunks of
// kSumChunk sorted tokens, whatever rows they belong to: an id that half the
// batch has is summed by as many workgroups as rare ones.  A run of tokens that
// ends in the next chunk at the latest is summed where it starts and its row
// written at once; a longer one leaves one partial row per chunk, and a last
// kernel adds those in order.  No atomics but on counters in shared memory.  The sums are bound by HBM
// (16384 bfloat16 tokens over 50257 x 2048, every row written: 273 MB in 50 us, 5.4
// TB/s), the sort, merge and join by the latency of a few dependent round trips
// (10 us each).
#include "lookup_kernel.h"

#include <algorithm>

#include "launch.h"
#include "micro_sparsify.h"
#include "value_types.h"

namespace micro {
namespace {

constexpr int kBlock = 256;

__device__ __forceinline__ int64_t token_id(const TokenIds& ids, int64_t t) {
    return ids.wide ? static_cast<const int64_t*>(ids.at)[t] : static_cast<const int32_t*>(ids.at)[t];
}

// A group of 2^group_bits threads takes a row; each thread `kVec` adjacent
// values at a time, 16 bytes where the type has 2- or 4-byte values.
template <class T>
__global__ __launch_bounds__(kBlock) void lookup_kernel(const T* table, int64_t table_stride, int64_t vocab, int32_t dim,
                                                        TokenIds ids, int64_t tokens, float scale, T* out,
                                                        int64_t out_stride, int group_bits) {
    constexpr int kVec = 16 / sizeof(T);
    const int group = 1 << group_bits, lane = threadIdx.x & (group - 1);
    const int64_t t = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) >> group_bits;
    if (t >= tokens) return;
    const int64_t id = token_id(ids, t);
    const bool known = id >= 0 && id < vocab;
    const T* row = table + (known ? id : 0) * table_stride;
    T* to = out + t * out_stride;
    const float factor = known ? scale : __builtin_nanf("");
    int c = lane * kVec;
    for (; c + kVec <= dim; c += group * kVec) {
        float x[kVec];
        load_floats<T, kVec>(row + c, x);
#pragma unroll
        for (int j = 0; j < kVec; ++j) x[j] *= factor;
        store_floats<T, kVec>(to + c, x);
    }
    for (; c < dim; ++c) to[c] = rounded<T>(static_cast<float>(row[c]) * factor);
}

// ---------------------------------------------------------------------------
// the order: positions sorted by id, stable
// ---------------------------------------------------------------------------

constexpr int kSortBlock = 1024, kSortWaves = kSortBlock / 64;
constexpr int kSortRounds = kSortTile / kSortBlock;
constexpr int kDigitBits = 8, kDigits = 1 << kDigitBits;

struct SortShared {
    uint32_t keys[kSortTile];
    uint16_t at[kSortTile];                  // positions in the tile, in the order so far
    uint32_t first[kSortWaves][kDigits];     // of a wave's run of a digit
    uint32_t totals[kDigits];
};

// Sorts n <= kSortTile keys of one tile with `passes` stable passes of
// kDigitBits each.  Every wave owns an equal run of the tile, 64 entries a
// round, all rounds in registers: the lanes of one digit find each other by a
// match over the wave, one of them adds their number to the wave's counter of
// the digit, and what it held before is the group's place in the wave's run of
// that digit.  A scan over (digit, wave) turns counters into places.
template <int kRounds>
__device__ void sort_passes(SortShared& s, int n, int passes) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int base = wave * kRounds * 64;
    for (int i = threadIdx.x; i < n; i += kSortBlock) s.at[i] = static_cast<uint16_t>(i);
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * kDigitBits;
        for (int i = threadIdx.x; i < kSortWaves * kDigits; i += kSortBlock) (&s.first[0][0])[i] = 0;
        __syncthreads();
        uint32_t at[kRounds], digit[kRounds], place[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = base + r * 64 + lane;
            at[r] = s.at[i < n ? i : 0];
        }
#pragma unroll
        for (int r = 0; r < kRounds; ++r) digit[r] = (s.keys[at[r]] >> shift) & (kDigits - 1);
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const bool in = base + r * 64 + lane < n;
            const uint64_t ins = __ballot(in);
            uint32_t low = static_cast<uint32_t>(ins), high = static_cast<uint32_t>(ins >> 32);
#pragma unroll
            for (int b = 0; b < kDigitBits; ++b) {
                const uint32_t bit = 0u - ((digit[r] >> b) & 1);  // all ones where it is set
                const uint64_t set = __ballot(bit != 0);
                low &= ~(static_cast<uint32_t>(set) ^ bit);
                high &= ~(static_cast<uint32_t>(set >> 32) ^ bit);
            }
            const uint64_t same = static_cast<uint64_t>(high) << 32 | low;
            const int leader = in ? __ffsll(static_cast<unsigned long long>(same)) - 1 : lane;
            uint32_t held = 0;
            if (in && lane == leader) held = atomicAdd(&s.first[wave][digit[r]], static_cast<uint32_t>(__popcll(same)));
            place[r] = __shfl(held, leader) + __popcll(same & ((uint64_t(1) << lane) - 1));
        }
        __syncthreads();
        // counts to places: within a digit by wave, digits in order
        if (threadIdx.x < kDigits) {
            uint32_t c[kSortWaves], sum = 0;
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) c[w] = s.first[w][threadIdx.x];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                s.first[w][threadIdx.x] = sum;
                sum += c[w];
            }
            s.totals[threadIdx.x] = sum;
        }
        __syncthreads();
        if (wave == 0) {  // exclusive scan of the digits' totals, kDigits / 64 a lane
            uint32_t own[kDigits / 64], sum = 0;
            for (int j = 0; j < kDigits / 64; ++j) {
                own[j] = sum;
                sum += s.totals[lane * (kDigits / 64) + j];
            }
            uint32_t up = sum;
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t x = __shfl_up(up, d);
                if (lane >= d) up += x;
            }
            for (int j = 0; j < kDigits / 64; ++j) s.totals[lane * (kDigits / 64) + j] = up - sum + own[j];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
            if (base + r * 64 + lane < n)
                s.at[s.totals[digit[r]] + s.first[wave][digit[r]] + place[r]] = static_cast<uint16_t>(at[r]);
        __syncthreads();
    }
}

__device__ void sort_tile(SortShared& s, int n, int passes) {
    if (n <= kSortBlock)
        sort_passes<1>(s, n, passes);
    else
        sort_passes<kSortRounds>(s, n, passes);
}

// Ids that a thread has in flight.
constexpr int kIdsAhead = kSortRounds;

// A workgroup sorts a tile of kSortTile tokens.  Ids without a part get the key
// `vocab`, behind all others.
__global__ __launch_bounds__(kSortBlock) void sort_kernel(TokenIds ids, int64_t tokens, int64_t vocab, int64_t padding,
                                                          int passes, uint32_t* keys, uint32_t* order) {
    __shared__ SortShared s;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kSortTile;
    const int n = static_cast<int>(tokens - first < kSortTile ? tokens - first : kSortTile);
    for (int i = threadIdx.x; i < n; i += kIdsAhead * kSortBlock) {
        int64_t id[kIdsAhead];
#pragma unroll
        for (int u = 0; u < kIdsAhead; ++u)
            id[u] = token_id(ids, first + (i + u * kSortBlock < n ? i + u * kSortBlock : n - 1));
#pragma unroll
        for (int u = 0; u < kIdsAhead; ++u)
            if (i + u * kSortBlock < n)
                s.keys[i + u * kSortBlock] =
                    static_cast<uint32_t>(id[u] < 0 || id[u] >= vocab || id[u] == padding ? vocab : id[u]);
    }
    __syncthreads();
    sort_tile(s, n, passes);
    for (int i = threadIdx.x; i < n; i += kSortBlock) {
        const uint32_t at = s.at[i];
        keys[first + i] = s.keys[at];
        order[first + i] = static_cast<uint32_t>(first + at);
    }
}

// The same order for calls of up to kMostRanked tokens, by many workgroups: each
// takes kRanked tokens of a tile and counts the keys of the tile that come before
// each (smaller ones, and equal ones at earlier positions), kRankLanes lanes a
// token and a sixteenth of the keys a wavefront.  More work than the sort, but
// without its chain of passes: whole calls of 3851 tokens by 144 took 19.8 us for
// 24.7, of 8190 by 192 32.6 for 36.2; at 16384 tokens it is 0.9 us slower.
constexpr int kRanked = 16, kRankLanes = 64 / kRanked;
constexpr int64_t kMostRanked = 8192;
static_assert(kSortTile % (kSortWaves * kRankLanes * 4) == 0 && kSortTile % kRanked == 0, "four keys a lane a step");

__global__ __launch_bounds__(kSortBlock) void rank_kernel(TokenIds ids, int64_t tokens, int64_t vocab, int64_t padding,
                                                          uint32_t* keys, uint32_t* order) {
    using Keys = uint32_t __attribute__((ext_vector_type(4)));
    __shared__ __attribute__((aligned(16))) uint32_t tile[kSortTile];
    __shared__ uint32_t counts[kSortWaves][64];
    const int64_t of_block = static_cast<int64_t>(blockIdx.x) * kRanked, first = of_block / kSortTile * kSortTile;
    const int n = static_cast<int>(tokens - first < kSortTile ? tokens - first : kSortTile);
    constexpr int kStep = kSortWaves * kRankLanes * 4;  // keys
    const int steps = (n + kStep - 1) / kStep;          // of every wavefront
    int64_t id[kSortRounds];
#pragma unroll
    for (int u = 0; u < kSortRounds; ++u) {
        const int i = threadIdx.x + u * kSortBlock;
        id[u] = token_id(ids, first + (i < n ? i : n - 1));
    }
#pragma unroll
    for (int u = 0; u < kSortRounds; ++u) {
        const int i = threadIdx.x + u * kSortBlock;
        // (places behind the last token come before no key)
        tile[i] = i >= n ? 0xffffffffu : static_cast<uint32_t>(id[u] < 0 || id[u] >= vocab || id[u] == padding ? vocab : id[u]);
    }
    __syncthreads();
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int at = static_cast<int>(of_block - first) + lane % kRanked;
    const uint32_t key = tile[at];
    uint32_t before = 0;
#pragma unroll 4
    for (int s = 0; s < steps; ++s) {
        const int j = ((wave * steps + s) * kRankLanes + lane / kRanked) * 4;
        const Keys other = *reinterpret_cast<const Keys*>(tile + j);
        const uint32_t bound = key + (j + 3 < at);  // (keys end below 2^31)
#pragma unroll
        for (int u = 0; u < 4; ++u) before += other[u] < bound;
        if (static_cast<uint32_t>(at - j) < 4)
#pragma unroll
            for (int u = 0; u < 3; ++u) before += j + u < at && other[u] == key;
    }
    counts[wave][lane] = before;
    __syncthreads();
    if (threadIdx.x >= kRanked || at >= n) return;
    uint32_t rank = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w)
#pragma unroll
        for (int l = 0; l < kRankLanes; ++l) rank += counts[w][l * kRanked + lane];
    keys[first + rank] = key;
    order[first + rank] = static_cast<uint32_t>(first + at);
}

// Merges up to kMergeRuns neighbouring sorted runs of `run` entries: an entry's
// place is its own rank plus the entries of each other run that come before it
// (equal keys of an earlier run do, those of a later one do not).  Each run is
// searched in two steps: among kSamples of its keys, evenly spaced, which the
// workgroup keeps in shared memory, then between two of them.  (Binary searches
// in global memory alone took three times as long for eight runs.)
constexpr int kMergeRuns = 8, kSamples = 256;
static_assert(kSortTile % kSamples == 0, "samples of a run");

__global__ __launch_bounds__(kBlock) void merge_kernel(const uint32_t* keys, const uint32_t* order, int64_t n, int64_t run,
                                                       uint32_t* to_keys, uint32_t* to_order) {
    __shared__ uint32_t samples[kMergeRuns][kSamples];
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
    // a workgroup's entries are of one run
    const int64_t group = static_cast<int64_t>(blockIdx.x) * kBlock / (kMergeRuns * run) * (kMergeRuns * run);
    const int64_t spacing = run / kSamples;
    static_assert(kBlock == kSamples, "a sample a thread");
    uint32_t sample[kMergeRuns];
#pragma unroll
    for (int q = 0; q < kMergeRuns; ++q) {
        const int64_t at = group + q * run + (threadIdx.x + 1) * spacing - 1;
        sample[q] = keys[at < n ? at : n - 1];
        if (at >= n) sample[q] = 0xffffffffu;
    }
    const uint32_t key = keys[i < n ? i : n - 1];
#pragma unroll
    for (int q = 0; q < kMergeRuns; ++q) samples[q][threadIdx.x] = sample[q];
    __syncthreads();
    if (i >= n) return;
    const int own = static_cast<int>((i - group) / run);
    const auto precedes = [&](int q, uint32_t other) { return q < own ? other <= key : other < key; };
    int64_t before[kMergeRuns], end[kMergeRuns];  // how many of a run come before: between these
#pragma unroll
    for (int q = 0; q < kMergeRuns; ++q) {
        const int64_t start = group + q * run, length = q == own || start >= n ? 0 : n - start < run ? n - start : run;
        int windows = 0;
#pragma unroll
        for (int step = kSamples / 2; step > 0; step /= 2)
            if (precedes(q, samples[q][windows + step - 1])) windows += step;
        if (precedes(q, samples[q][windows])) ++windows;  // all of them
        before[q] = windows * spacing < length ? windows * spacing : length;
        end[q] = before[q] + spacing - 1 < length ? before[q] + spacing - 1 : length;
    }
    for (int64_t step = spacing / 2; step > 0; step /= 2) {
#pragma unroll
        for (int q = 0; q < kMergeRuns; ++q) {
            const bool in = before[q] + step <= end[q];
            const uint32_t other = keys[in ? group + q * run + before[q] + step - 1 : i];
            if (in && precedes(q, other)) before[q] += step;
        }
    }
    int64_t place = i - own * run;
#pragma unroll
    for (int q = 0; q < kMergeRuns; ++q) place += before[q];
    to_keys[place] = key;
    to_order[place] = order[i];
}

// ---------------------------------------------------------------------------
// the sums
// ---------------------------------------------------------------------------

template <class T, int kVec>
__device__ __forceinline__ void load_row(const T* row, int c, int dim, float (&x)[kVec]) {
    if (c + kVec <= dim) {
        load_floats<T, kVec>(row + c, x);
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) x[j] = c + j < dim ? static_cast<float>(row[c + j]) : 0.0f;
    }
}

template <class T, int kVec>
__device__ __forceinline__ void write_row(T* row, int c, int dim, const float (&sum)[kVec], float scale, bool accumulate) {
    float x[kVec];
    if (accumulate) {
        load_row<T, kVec>(row, c, dim, x);
#pragma unroll
        for (int j = 0; j < kVec; ++j) x[j] += scale * sum[j];
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) x[j] = scale * sum[j];
    }
    if (c + kVec <= dim) {
        store_floats<T, kVec>(row + c, x);
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            if (c + j < dim) row[c + j] = rounded<T>(x[j]);
    }
}

template <int kVec>
__device__ __forceinline__ void write_partial(float* row, int c, int dim, const float (&sum)[kVec]) {
    if (c + kVec <= dim) {
        store_floats<float, kVec>(row + c, sum);
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            if (c + j < dim) row[c + j] = sum[j];
    }
}

// Rows that a thread has in flight.
constexpr int kRowsAhead = 8;

// Raw vectors: a row's values stay as they were read until they are added.
template <class T, int kVec>
__device__ __forceinline__ Pack<T, kVec> load_raw(const T* row, int c, int dim) {
    Pack<T, kVec> x;
    if (c + kVec <= dim) {
        x = *reinterpret_cast<const Pack<T, kVec>*>(row + c);
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) x.v[j] = c + j < dim ? row[c + j] : static_cast<T>(0.0f);
    }
    return x;
}

// First entry of the sorted keys that is not below `key`.
__device__ int64_t lower_bound(const uint32_t* keys, int64_t n, uint32_t key) {
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t m = lo + (hi - lo) / 2;
        if (keys[m] < key)
            lo = m + 1;
        else
            hi = m;
    }
    return lo;
}

constexpr int kZeroRowsMax = 256;

// Zeros into those of `rows` rows from `from` on that no token has.
template <class T>
__device__ void zero_absent(const uint32_t* keys, int64_t tokens, int64_t from, int rows, T* table, int64_t stride, int32_t dim) {
    constexpr int kVec = 16 / sizeof(T);
    __shared__ uint32_t present[kZeroRowsMax];
    __shared__ int64_t range[2];
    for (int r = threadIdx.x; r < rows; r += kBlock) present[r] = 0;
    if (threadIdx.x < 2)
        range[threadIdx.x] = lower_bound(keys, tokens, static_cast<uint32_t>(from + (threadIdx.x == 0 ? 0 : rows)));
    __syncthreads();
    for (int64_t i = range[0] + threadIdx.x; i < range[1]; i += kBlock) present[keys[i] - from] = 1;
    __syncthreads();
    const int vectors = (dim + kVec - 1) / kVec;
    // past the cache, where they would push out the rows that are being summed:
    // 50257 x 2048 bfloat16, 87 us a call against 111
    const float zeros[kVec] = {};
    for (int i = threadIdx.x; i < rows * vectors; i += kBlock) {
        const int r = i / vectors, c = (i - r * vectors) * kVec;
        if (present[r]) continue;
        T* at = table + (from + r) * stride + c;
        if (c + kVec <= dim) {
            stream_floats<T, kVec>(at, zeros);
        } else {
            for (int j = 0; c + j < dim; ++j) at[j] = static_cast<T>(0.0f);
        }
    }
}

// A group of 2^group_bits threads, whole wavefronts, takes a chunk of kSumChunk
// sorted tokens, columns [c, c + kVec) a thread.  Keys and positions are the same
// for a wavefront: a lane each holds them.  (Narrow rows leave lanes idle; groups
// of fewer lanes, which had to load every key, took 40 us for a whole call of
// 8190 tokens by 192 against 36, both with the order from the sort.)
// A run (the tokens of one row) belongs to the chunk that it starts in, which
// sums it to its end where that lies in the next chunk at the latest.  Of a
// longer run each chunk leaves a partial row: chunk q's part of a run that comes
// in from the chunk before goes to row 2q, of one that starts in it to row
// 2q + 1.  The workgroups from `sums` on write the rows without a token,
// zero_rows each: beside the sums, so that every row is written once.
template <class T>
__global__ __launch_bounds__(kBlock) void sum_kernel(const T* grad, int64_t grad_stride, int64_t tokens, const uint32_t* keys,
                                                     const uint32_t* order, uint32_t vocab, float scale, bool accumulate,
                                                     T* table, int64_t table_stride, int32_t dim, float* partials,
                                                     int group_bits, uint32_t sums, int zero_rows) {
    constexpr int kVec = 16 / sizeof(T), C = kSumChunk;
    if (blockIdx.x >= sums) {
        const int64_t from = static_cast<int64_t>(blockIdx.x - sums) * zero_rows;
        const int rows = static_cast<int>(vocab - from < zero_rows ? vocab - from : zero_rows);
        if (blockIdx.y == 0) zero_absent(keys, tokens, from, rows, table, table_stride, dim);
        return;
    }
    const int group = 1 << group_bits, lane = threadIdx.x & (group - 1);
    const int in_block = static_cast<int>(threadIdx.x) >> group_bits;
    const int64_t chunk = static_cast<int64_t>(blockIdx.x) * (kBlock >> group_bits) +
                          __builtin_amdgcn_readfirstlane(in_block);
    const int64_t first = chunk * C;
    const int c = (static_cast<int>(blockIdx.y) * group + lane) * kVec;
    // (lanes behind a row's end stay: the others read keys from them)
    if (first >= tokens || c - (lane & 63) * kVec >= dim) return;
    const int64_t rest = tokens - first;
    const int n = static_cast<int>(rest < C ? rest : C);
    // this chunk's entries, the next one's and one more
    const int l = threadIdx.x & 63;
    const uint32_t held_key = keys[first + (l < rest ? l : rest - 1)];
    const uint32_t held_at = order[first + (l < rest ? l : rest - 1)];
    const uint32_t before = keys[first > 0 ? first - 1 : 0], earlier = keys[first > C ? first - C - 1 : 0];
    static_assert(2 * C < 64, "a lane an entry");
    const auto key_of = [&](int i) -> uint32_t { return __builtin_amdgcn_readlane(held_key, i); };  // i < rest
    const auto at_of = [&](int i) -> int64_t { return static_cast<uint32_t>(__builtin_amdgcn_readlane(held_at, i)); };
    const uint32_t head = key_of(0), tail = key_of(n - 1);
    const bool from_before = first > 0 && before == head;
    const bool into_next = n < rest && key_of(n) == tail;
    int start = 0, end = n;
    bool open_start = from_before, open_end = into_next;
    if (from_before && (first == C || earlier != head) && !(tail == head && into_next)) {
        // it started in the chunk before, which sums it to its end
        open_start = false;
        while (start < n && key_of(start) == head) ++start;
    }
    if (into_next && !(from_before && tail == head) && (2 * C >= rest || key_of(2 * C) != tail)) {
        // it starts here and ends in the next chunk
        open_end = false;
        while (end < rest && end < 2 * C && key_of(end) == tail) ++end;
    }
    const auto load = [&](int b, Pack<T, kVec> (&x)[kRowsAhead]) {
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u)
            x[u] = load_raw<T, kVec>(grad + at_of(b + u < end ? b + u : end - 1) * grad_stride, c, dim);
    };
    float sum[kVec] = {};
    int run = start;  // where the run being summed began
    const auto add = [&](int b, const Pack<T, kVec> (&x)[kRowsAhead]) {
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            const int i = b + u;
            if (i >= end) break;
#pragma unroll
            for (int j = 0; j < kVec; ++j) sum[j] += static_cast<float>(x[u].v[j]);
            const uint32_t key = key_of(i);
            if (i != end - 1 && key_of(i + 1) == key) continue;
            if (key < vocab) {
                const bool in = run == 0 && open_start, out = i == end - 1 && open_end;
                if (!in && !out)
                    write_row<T, kVec>(table + key * table_stride, c, dim, sum, scale, accumulate);
                else
                    write_partial<kVec>(partials + (2 * chunk + (in ? 0 : 1)) * dim, c, dim, sum);
            }
#pragma unroll
            for (int j = 0; j < kVec; ++j) sum[j] = 0.0f;
            run = i + 1;
        }
    };
    if (start >= end) return;
    Pack<T, kVec> even[kRowsAhead], odd[kRowsAhead];
    load(start, even);
#pragma unroll 1
    for (int b = start; b < end; b += 2 * kRowsAhead) {
        load(b + kRowsAhead, odd);
        add(b, even);
        if (b + 2 * kRowsAhead < end) load(b + 2 * kRowsAhead, even);
        add(b + kRowsAhead, odd);
    }
}

// Adds the partial rows of the run that starts in a chunk and goes on past the
// next one:
// 256 columns a workgroup, each wavefront a quarter of the run's chunks, the
// quarters in their order.
__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }

template <class T>
__global__ __launch_bounds__(kBlock) void join_kernel(int64_t tokens, const uint32_t* keys, uint32_t vocab, float scale,
                                                      bool accumulate, T* table, int64_t table_stride, int32_t dim,
                                                      const float* partials) {
    constexpr int kVec = 4, kParts = kBlock / 64;
    __shared__ float4 quarters[kParts][64];
    const int lane = threadIdx.x & 63, part = threadIdx.x >> 6;
    const int64_t chunk = blockIdx.x, first = chunk * kSumChunk, next = first + kSumChunk;
    if (next >= tokens) return;
    const uint32_t key = keys[next - 1], behind = keys[next], start = keys[first], ahead = keys[first > 0 ? first - 1 : 0];
    if (key >= vocab || behind != key) return;                 // no run goes on
    if (start == key && first > 0 && ahead == key) return;     // it started before this chunk
    // the run's last chunk: the last one that begins with its key
    int64_t last = chunk + 1;
    for (;; last += 64) {
        const int64_t at = (last + lane) * kSumChunk;
        const uint64_t other = __ballot(at >= tokens || keys[at < tokens ? at : tokens - 1] != key);
        if (other != 0) {
            last += __ffsll(static_cast<unsigned long long>(other)) - 2;
            break;
        }
    }
    if (last == chunk + 1) return;                             // summed by the chunk it starts in
    const int64_t each = (last - chunk + kParts) / kParts;                   // chunks [chunk, last] in parts
    const int64_t from = chunk + part * each, until = from + each - 1 < last ? from + each - 1 : last;
    const int c = (static_cast<int>(blockIdx.y) * 64 + lane) * kVec;
    float sum[kVec] = {};
    if (c < dim)
        for (int64_t q = from; q <= until; q += kRowsAhead) {
            float x[kRowsAhead][kVec];
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) {
                const int64_t at = q + u <= until ? q + u : until;
                load_row<float, kVec>(partials + (2 * at + (at == chunk ? 1 : 0)) * dim, c, dim, x[u]);
            }
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u)
                if (q + u <= until)
#pragma unroll
                    for (int j = 0; j < kVec; ++j) sum[j] += x[u][j];
        }
    quarters[part][lane] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    __syncthreads();
    if (part != 0 || c >= dim) return;
    float4 all = quarters[0][lane];
    for (int w = 1; w < kParts; ++w) all = add4(all, quarters[w][lane]);
    const float total[kVec] = {all.x, all.y, all.z, all.w};
    write_row<T, kVec>(table + key * table_stride, c, dim, total, scale, accumulate);
}

// log2 of the threads that share a row of `vectors` vectors.
int group_bits_for(int64_t vectors, int most) {
    int bits = 0;
    while (bits < most && (int64_t(1) << bits) < vectors) ++bits;
    return bits;
}

template <class T>
hipError_t lookup(const Rows& table, int64_t vocab, int32_t dim, const TokenIds& ids, int64_t tokens, float scale,
                  const Rows& out, hipStream_t stream) {
    constexpr int kVec = 16 / sizeof(T);
    const int bits = group_bits_for((dim + kVec - 1) / kVec, 8);
    const int64_t per_block = kBlock >> bits;
    return launch(lookup_kernel<T>, dim3(static_cast<uint32_t>((tokens + per_block - 1) / per_block)), dim3(kBlock), stream,
                  static_cast<const T*>(table.at), table.stride, vocab, dim, ids, tokens, scale, static_cast<T*>(out.at),
                  out.stride, bits);
}

template <class T>
hipError_t sums(const Rows& grad, int64_t tokens, float scale, bool accumulate, const Rows& table, int64_t vocab,
                int32_t dim, const uint32_t* keys, const uint32_t* order, float* partials, hipStream_t stream) {
    constexpr int kVec = 16 / sizeof(T);
    const int64_t chunks = (tokens + kSumChunk - 1) / kSumChunk;
    const auto grid = [&](int bits, int vec) {
        const int64_t per_block = kBlock >> bits;
        return dim3(static_cast<uint32_t>((chunks + per_block - 1) / per_block),
                    static_cast<uint32_t>((dim + (vec << bits) - 1) / (vec << bits)));
    };
    const int bits = std::max(group_bits_for((dim + kVec - 1) / kVec, 8), 6);
    dim3 blocks = grid(bits, kVec);
    const uint32_t summing = blocks.x;
    // 64 KB of rows a zeroing workgroup
    const int zero_rows = static_cast<int>(std::clamp<int64_t>(65536 / (dim * int64_t(sizeof(T))), 1, kZeroRowsMax));
    if (!accumulate) blocks.x += static_cast<uint32_t>((vocab + zero_rows - 1) / zero_rows);
    const hipError_t e = launch(sum_kernel<T>, blocks, dim3(kBlock), stream, static_cast<const T*>(grad.at), grad.stride, tokens,
                                keys, order, static_cast<uint32_t>(vocab), scale, accumulate, static_cast<T*>(table.at),
                                table.stride, dim, partials, bits, summing, zero_rows);
    if (e != hipSuccess || chunks < 2) return e;
    return launch(join_kernel<T>, dim3(static_cast<uint32_t>(chunks), static_cast<uint32_t>((dim + 255) / 256)), dim3(kBlock),
                  stream, tokens, keys, static_cast<uint32_t>(vocab), scale, accumulate, static_cast<T*>(table.at),
                  table.stride, dim, partials);
}

}  // namespace

hipError_t launch_lookup(const Rows& table, int64_t vocab, int32_t dim, const TokenIds& ids, int64_t tokens,
                         float scale, const Rows& out, hipStream_t stream) {
    if (tokens == 0) return hipSuccess;
    if (table.type == MICRO_TYPE_F32) return lookup<float>(table, vocab, dim, ids, tokens, scale, out, stream);
    if (table.type == MICRO_TYPE_F16) return lookup<f16>(table, vocab, dim, ids, tokens, scale, out, stream);
    return lookup<bf16>(table, vocab, dim, ids, tokens, scale, out, stream);
}

hipError_t launch_lookup_grad(const Rows& grad, int64_t tokens, const TokenIds& ids, int64_t padding, float scale,
                              bool accumulate, const Rows& table, int64_t vocab, int32_t dim,
                              const LookupGradScratch& scratch, hipStream_t stream) {
    if (tokens == 0 && accumulate) return hipSuccess;
    int passes = 1;
    while (passes < 4 && (vocab >> (passes * kDigitBits)) != 0) ++passes;
    hipError_t e = hipSuccess;
    if (tokens > 0 && tokens <= kMostRanked) {
        e = launch(rank_kernel, dim3(static_cast<uint32_t>((tokens + kRanked - 1) / kRanked)), dim3(kSortBlock), stream, ids,
                   tokens, vocab, padding, scratch.keys[0], scratch.order[0]);
    } else if (tokens > 0) {
        e = launch(sort_kernel, dim3(static_cast<uint32_t>((tokens + kSortTile - 1) / kSortTile)), dim3(kSortBlock), stream,
                   ids, tokens, vocab, padding, passes, scratch.keys[0], scratch.order[0]);
    }
    if (e != hipSuccess) return e;
    int in = 0;
    for (int64_t run = kSortTile; run < tokens; run *= kMergeRuns, in ^= 1) {
        e = launch(merge_kernel, dim3(static_cast<uint32_t>((tokens + kBlock - 1) / kBlock)), dim3(kBlock), stream,
                   scratch.keys[in], scratch.order[in], tokens, run, scratch.keys[in ^ 1], scratch.order[in ^ 1]);
        if (e != hipSuccess) return e;
    }
    if (table.type == MICRO_TYPE_F32)
        return sums<float>(grad, tokens, scale, accumulate, table, vocab, dim, scratch.keys[in], scratch.order[in],
                           scratch.partials, stream);
    if (table.type == MICRO_TYPE_F16)
        return sums<f16>(grad, tokens, scale, accumulate, table, vocab, dim, scratch.keys[in], scratch.order[in],
                         scratch.partials, stream);
    return sums<bf16>(grad, tokens, scale, accumulate, table, vocab, dim, scratch.keys[in], scratch.order[in],
                      scratch.partials, stream);
}

}  // namespace micro

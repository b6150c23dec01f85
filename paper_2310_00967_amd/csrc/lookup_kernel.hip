// gfx950 kernels of the token table: the lookup of rows with scaling, and its
// gradient by sorted tokens.
//   lookup    out[t] = scale * table[ids[t]]: a gather, bound by HBM.
//   gradient  table[v] (+)= scale * sum of grad[t] over the tokens with id v.
// The gradient's tokens are sorted by id (stably, so a row's terms keep their
// order and the binary32 sum is the same on every run) and cut into chunks of
// kSumChunk sorted tokens, whatever rows they belong to: an id that half the
// batch has is summed by as many workgroups as rare ones.  A row whose run of
// tokens ends inside its chunk is written at once; a run across chunks leaves
// one partial row per chunk, and a second kernel adds those in order.  No
// atomics.
#include "lookup_kernel.h"
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
            uint64_t same = __ballot(in);
#pragma unroll
            for (int b = 0; b < kDigitBits; ++b) {
                const bool bit = (digit[r] >> b) & 1;
                const uint64_t set = __ballot(bit);
                same &= bit ? set : ~set;
            }
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
    else if (n <= kSortTile / 4)
        sort_passes<kSortRounds / 4>(s, n, passes);
    else
        sort_passes<kSortRounds>(s, n, passes);
}

// The first workgroups sort one tile of kSortTile tokens each; the others
// (where every row is to be written) fill the table with zeros meanwhile.
// Ids without a part get the key `vocab`, behind all others.
__global__ __launch_bounds__(kSortBlock) void sort_kernel(TokenIds ids, int64_t tokens, int64_t vocab, int64_t padding,
                                                          int passes, uint32_t tiles, uint32_t* keys, uint32_t* order,
                                                          char* table, int64_t row_bytes, int64_t stride_bytes) {
    __shared__ SortShared s;
    if (blockIdx.x < tiles) {
        const int64_t first = static_cast<int64_t>(blockIdx.x) * kSortTile;
        const int n = static_cast<int>(tokens - first < kSortTile ? tokens - first : kSortTile);
        for (int i = threadIdx.x; i < n; i += kSortBlock) {
            const int64_t id = token_id(ids, first + i);
            s.keys[i] = static_cast<uint32_t>(id < 0 || id >= vocab || id == padding ? vocab : id);
        }
        __syncthreads();
        sort_tile(s, n, passes);
        for (int i = threadIdx.x; i < n; i += kSortBlock) {
            const uint32_t at = s.at[i];
            keys[first + i] = s.keys[at];
            order[first + i] = static_cast<uint32_t>(first + at);
        }
        return;
    }
    const int64_t fillers = gridDim.x - tiles, filler = blockIdx.x - tiles;
    if (stride_bytes == row_bytes) {  // one run of bytes
        const int64_t bytes = vocab * row_bytes, head = (16 - (reinterpret_cast<uintptr_t>(table) & 15)) & 15;
        const int64_t vectors = bytes > head ? (bytes - head) / 16 : 0;
        uint4* v = reinterpret_cast<uint4*>(table + head);
        for (int64_t i = filler * kSortBlock + threadIdx.x; i < vectors; i += fillers * kSortBlock)
            v[i] = make_uint4(0, 0, 0, 0);
        if (filler == 0) {
            uint16_t* ends = reinterpret_cast<uint16_t*>(table);
            const int64_t done = head + vectors * 16;
            for (int64_t i = threadIdx.x; 2 * i < (head < bytes ? head : bytes); i += kSortBlock) ends[i] = 0;
            for (int64_t i = done / 2 + threadIdx.x; 2 * i < bytes; i += kSortBlock) ends[i] = 0;
        }
    } else {
        for (int64_t r = filler; r < vocab; r += fillers) {
            uint16_t* row = reinterpret_cast<uint16_t*>(table + r * stride_bytes);
            for (int64_t i = threadIdx.x; 2 * i < row_bytes; i += kSortBlock) row[i] = 0;
        }
    }
}

// Merges neighbouring sorted runs of `run` entries: an entry's place is its
// own rank plus the entries of the sibling run that come before it (equal keys
// of the left run do, those of the right run do not).
__global__ __launch_bounds__(kBlock) void merge_kernel(const uint32_t* keys, const uint32_t* order, int64_t n, int64_t run,
                                                       uint32_t* to_keys, uint32_t* to_order) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
    if (i >= n) return;
    const int64_t pair = i / (2 * run) * (2 * run), middle = pair + run < n ? pair + run : n;
    const int64_t end = pair + 2 * run < n ? pair + 2 * run : n;
    const uint32_t key = keys[i];
    const bool left = i < middle;
    int64_t lo = left ? middle : pair, hi = left ? end : middle;
    const int64_t sibling = lo;
    while (lo < hi) {
        const int64_t m = lo + (hi - lo) / 2;
        if (left ? keys[m] < key : keys[m] <= key)
            lo = m + 1;
        else
            hi = m;
    }
    const int64_t own = left ? i - pair : i - middle;
    to_keys[pair + own + (lo - sibling)] = key;
    to_order[pair + own + (lo - sibling)] = order[i];
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
#pragma unroll
    for (int j = 0; j < kVec; ++j)
        if (c + j < dim) row[c + j] = sum[j];
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

// A group of 2^group_bits threads takes a chunk of kSumChunk sorted tokens,
// columns [c, c + kVec) a thread.  kWide: groups of whole wavefronts, whose
// keys and positions are the same in every lane and stay in scalar registers.
// Partial rows: chunk q's run that comes in from the chunk before (or covers
// the whole chunk) goes to row 2q, one that starts in it and goes on into the
// next to row 2q + 1.
template <class T, bool kWide>
__global__ __launch_bounds__(kBlock) void sum_kernel(const T* grad, int64_t grad_stride, int64_t tokens, const uint32_t* keys,
                                                     const uint32_t* order, uint32_t vocab, float scale, bool accumulate,
                                                     T* table, int64_t table_stride, int32_t dim, float* partials,
                                                     int group_bits) {
    constexpr int kVec = 16 / sizeof(T);
    const int group = 1 << group_bits, lane = threadIdx.x & (group - 1);
    const int in_block = static_cast<int>(threadIdx.x) >> group_bits;
    const int64_t chunk = static_cast<int64_t>(blockIdx.x) * (kBlock >> group_bits) +
                          (kWide ? __builtin_amdgcn_readfirstlane(in_block) : in_block);
    const int64_t first = chunk * kSumChunk;
    const int c = (static_cast<int>(blockIdx.y) * group + lane) * kVec;
    if (first >= tokens || c >= dim) return;
    const int n = static_cast<int>(tokens - first < kSumChunk ? tokens - first : kSumChunk);
    const bool from_before = first > 0 && keys[first - 1] == keys[first];
    const bool into_next = first + n < tokens && keys[first + n] == keys[first + n - 1];
    const auto load = [&](int b, Pack<T, kVec> (&x)[kRowsAhead]) {
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u)
            x[u] = load_raw<T, kVec>(grad + order[first + (b + u < n ? b + u : n - 1)] * grad_stride, c, dim);
    };
    float sum[kVec] = {};
    int start = 0;  // of the run being summed
    const auto add = [&](int b, const Pack<T, kVec> (&x)[kRowsAhead]) {
        uint32_t key[kRowsAhead + 1];
#pragma unroll
        for (int u = 0; u <= kRowsAhead; ++u) key[u] = keys[first + (b + u < n ? b + u : n - 1)];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u) {
            const int i = b + u;
            if (i >= n) break;
#pragma unroll
            for (int j = 0; j < kVec; ++j) sum[j] += static_cast<float>(x[u].v[j]);
            const bool ends = i == n - 1 || key[u + 1] != key[u];
            if (!ends) continue;
            if (key[u] < vocab) {
                const bool open_start = start == 0 && from_before, open_end = i == n - 1 && into_next;
                if (!open_start && !open_end)
                    write_row<T, kVec>(table + key[u] * table_stride, c, dim, sum, scale, accumulate);
                else
                    write_partial<kVec>(partials + (2 * chunk + (open_start ? 0 : 1)) * dim, c, dim, sum);
            }
#pragma unroll
            for (int j = 0; j < kVec; ++j) sum[j] = 0.0f;
            start = i + 1;
        }
    };
    static_assert(kSumChunk % (2 * kRowsAhead) == 0, "batches of rows in pairs");
    Pack<T, kVec> even[kRowsAhead], odd[kRowsAhead];
    load(0, even);
#pragma unroll 1
    for (int b = 0; b < n; b += 2 * kRowsAhead) {
        load(b + kRowsAhead, odd);
        add(b, even);
        if (b + 2 * kRowsAhead < n) load(b + 2 * kRowsAhead, even);
        add(b + kRowsAhead, odd);
    }
}

// Adds the partial rows of the run that starts in a chunk and goes on past it.
template <class T>
__global__ __launch_bounds__(kBlock) void join_kernel(int64_t tokens, const uint32_t* keys, uint32_t vocab, float scale,
                                                      bool accumulate, T* table, int64_t table_stride, int32_t dim,
                                                      const float* partials, int group_bits) {
    constexpr int kVec = 4;
    const int group = 1 << group_bits, lane = threadIdx.x & (group - 1);
    const int64_t chunk = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) >> group_bits;
    const int64_t first = chunk * kSumChunk, next = first + kSumChunk;
    const int c = (static_cast<int>(blockIdx.y) * group + lane) * kVec;
    if (next >= tokens || c >= dim) return;
    const uint32_t key = keys[next - 1];
    if (key >= vocab || keys[next] != key) return;                           // no run goes on
    if (keys[first] == key && first > 0 && keys[first - 1] == key) return;   // it started before this chunk
    // the run's end
    int64_t lo = next, hi = tokens;
    while (lo < hi) {
        const int64_t m = lo + (hi - lo) / 2;
        if (keys[m] <= key)
            lo = m + 1;
        else
            hi = m;
    }
    const int64_t last = (lo - 1) / kSumChunk;
    float sum[kVec];
    load_row<float, kVec>(partials + (2 * chunk + 1) * dim, c, dim, sum);
    for (int64_t q = chunk + 1; q <= last; q += kRowsAhead) {
        float x[kRowsAhead][kVec];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u)
            load_row<float, kVec>(partials + 2 * (q + u <= last ? q + u : last) * dim, c, dim, x[u]);
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u)
            if (q + u <= last)
#pragma unroll
                for (int j = 0; j < kVec; ++j) sum[j] += x[u][j];
    }
    write_row<T, kVec>(table + key * table_stride, c, dim, sum, scale, accumulate);
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
    hipLaunchKernelGGL(lookup_kernel<T>, dim3(static_cast<uint32_t>((tokens + per_block - 1) / per_block)), dim3(kBlock),
                       0, stream, static_cast<const T*>(table.at), table.stride, vocab, dim, ids, tokens, scale,
                       static_cast<T*>(out.at), out.stride, bits);
    return hipGetLastError();
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
    const int bits = group_bits_for((dim + kVec - 1) / kVec, 8);
    const auto sum = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid(bits, kVec), dim3(kBlock), 0, stream, static_cast<const T*>(grad.at), grad.stride,
                           tokens, keys, order, static_cast<uint32_t>(vocab), scale, accumulate,
                           static_cast<T*>(table.at), table.stride, dim, partials, bits);
    };
    if (bits >= 6)
        sum(sum_kernel<T, true>);
    else
        sum(sum_kernel<T, false>);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || chunks < 2) return e;
    const int join_bits = group_bits_for((dim + 3) / 4, 6);
    hipLaunchKernelGGL(join_kernel<T>, grid(join_bits, 4), dim3(kBlock), 0, stream, tokens, keys,
                       static_cast<uint32_t>(vocab), scale, accumulate, static_cast<T*>(table.at), table.stride, dim,
                       partials, join_bits);
    return hipGetLastError();
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
    const int64_t size = table.type == MICRO_TYPE_F32 ? 4 : 2;
    int passes = 1;
    while (passes < 4 && (vocab >> (passes * kDigitBits)) != 0) ++passes;
    const uint32_t tiles = static_cast<uint32_t>((tokens + kSortTile - 1) / kSortTile);
    // a kilobyte and a half of the table a filling thread
    int64_t fillers = accumulate ? 0 : (vocab * dim * size) / (kSortBlock * 1536) + 1;
    if (fillers > 1024) fillers = 1024;
    hipLaunchKernelGGL(sort_kernel, dim3(tiles + static_cast<uint32_t>(fillers)), dim3(kSortBlock), 0, stream, ids,
                       tokens, vocab, padding, passes, tiles, scratch.keys[0], scratch.order[0],
                       static_cast<char*>(table.at), dim * size, table.stride * size);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || tokens == 0) return e;
    int in = 0;
    for (int64_t run = kSortTile; run < tokens; run *= 2, in ^= 1) {
        hipLaunchKernelGGL(merge_kernel, dim3(static_cast<uint32_t>((tokens + kBlock - 1) / kBlock)), dim3(kBlock), 0,
                           stream, scratch.keys[in], scratch.order[in], tokens, run, scratch.keys[in ^ 1],
                           scratch.order[in ^ 1]);
        if ((e = hipGetLastError()) != hipSuccess) return e;
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

// Shared by the handles of the language-model calls: their device scratch and
// the check that a call's arguments lie apart.
#pragma once

#include <algorithm>
#include <cstdint>

#include "host_util.h"
#include "strided_rows.h"

namespace micro {

inline int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Device memory cut into parts, each aligned to 256 bytes: first the sizes are
// added up, then one allocation is handed out in the same order.
struct Parts {
    char* base = nullptr;
    int64_t used = 0;
    template <class T>
    void take(T*& p, int64_t bytes) {
        p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += round_up(bytes, 256);
    }
};

// Allocates what `lay_out` takes, once.
template <class LayOut>
micro_status ensure(void** memory, const char* what, LayOut lay_out) {
    if (*memory) return MICRO_OK;
    Parts parts;
    lay_out(parts);
    void* p = nullptr;
    const hipError_t e = hipMalloc(&p, static_cast<size_t>(std::max<int64_t>(parts.used, 256)));
    if (e != hipSuccess) {
        forget_hip_error();
        lay_out(parts = Parts{});  // no part points anywhere
        set_thread_error("%s: %lld bytes of device scratch: %s", what, static_cast<long long>(parts.used),
                         hipGetErrorString(e));
        return e == hipErrorOutOfMemory ? MICRO_ENOMEM : MICRO_EHIP;
    }
    *memory = p;
    parts = Parts{static_cast<char*>(p), 0};
    lay_out(parts);
    return MICRO_OK;
}

struct Region {
    RowSpan rows;
    bool written;
};

template <int N>
micro_status check_apart(const Region (&r)[N]) {
    for (int i = 0; i < N; ++i)
        for (int j = i + 1; j < N; ++j)
            if ((r[i].written || r[j].written) && rows_share_bytes(r[i].rows, r[j].rows))
                return refuse("an output shares memory with another argument");
    return MICRO_OK;
}

// `values` values of `size` bytes one after the other.
inline RowSpan run_of(const void* at, int64_t values, int64_t size) { return {at, 1, values * size, values * size}; }

// `rows` rows of `width` values of `size` bytes.
inline micro_status check_strided(const void* at, int64_t stride, int64_t rows, int64_t width, int64_t size) {
    if (stride < width) return refuse("a row stride is below the width of a row");
    if (stride > (int64_t(1) << 32) || (stride > 0 && rows > (int64_t(1) << 56) / stride))
        return refuse("a row stride is above 2^32, or the rows end past 2^56 values");
    if (rows > 0 && width > 0 && (!at || !aligned_to(at, size))) return refuse("rows are NULL or not aligned to their type");
    return MICRO_OK;
}

}  // namespace micro

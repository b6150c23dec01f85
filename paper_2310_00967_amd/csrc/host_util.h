// Shared by the host sources of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "micro_sparsify.h"

namespace micro {

// Sets the calling thread's error message, which micro_last_error(NULL)
// returns.
void set_thread_error(const char* fmt, ...) __attribute__((format(printf, 1, 2)));

// Makes a handle's device current for the scope of a call and restores the
// caller's current device afterwards.
struct CallDevice {
    int previous = -1;
    bool switched = false;
    explicit CallDevice(int device) {
        if (device >= 0 && hipGetDevice(&previous) == hipSuccess && previous != device)
            switched = hipSetDevice(device) == hipSuccess;
    }
    ~CallDevice() {
        if (switched) (void)hipSetDevice(previous);
    }
    CallDevice(const CallDevice&) = delete;
    CallDevice& operator=(const CallDevice&) = delete;
};

inline micro_status refuse(const char* what) {
    set_thread_error("%s", what);
    return MICRO_EINVAL;
}

// An error that is returned to the caller is taken from the runtime's record of
// the thread, where the next call that looks there would report it again.
inline void forget_hip_error() { (void)hipGetLastError(); }

inline micro_status report_hip(hipError_t e, const char* what) {
    if (e == hipSuccess) return MICRO_OK;
    forget_hip_error();
    set_thread_error("%s failed: %s", what, hipGetErrorString(e));
    return e == hipErrorOutOfMemory ? MICRO_ENOMEM : MICRO_EHIP;
}

inline int64_t type_bytes(int32_t type) { return type == MICRO_TYPE_F32 ? 4 : 2; }

inline bool type_valid(int32_t type) {
    return type == MICRO_TYPE_F32 || type == MICRO_TYPE_F16 || type == MICRO_TYPE_BF16;
}

inline bool aligned_to(const void* p, int64_t bytes) {
    return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0;
}

// Whether [a, a + an) and [b, b + bn), both in bytes, share a byte.
inline bool share_bytes(const void* a, int64_t an, const void* b, int64_t bn) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return an > 0 && bn > 0 && a0 < b0 + static_cast<uintptr_t>(bn) && b0 < a0 + static_cast<uintptr_t>(an);
}

}  // namespace micro

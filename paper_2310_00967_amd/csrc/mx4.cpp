// Host side of the microscaled 4-bit entry points (micro_mx4_*).
#include <new>

#include "handle_util.h"
#include "micro_sparsify.h"
#include "mx4_kernel.h"

struct micro_mx4 {
    int device = -1, compute_units = 256;
    hipStream_t stream = nullptr;
    void* memory = nullptr;  // the parts of products
    float* parts = nullptr;
};

namespace {

using namespace micro;

constexpr int64_t kMostSide = int64_t(1) << 24;

int64_t groups_of(int64_t cols) { return (cols + kMxGroup - 1) / kMxGroup; }

micro_status check_sides(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0) return refuse("a side is negative");
    if (rows > kMostSide || cols > kMostSide) {
        set_thread_error("a matrix of %lld x %lld: sides are at most 2^24", static_cast<long long>(rows),
                         static_cast<long long>(cols));
        return MICRO_ERANGE;
    }
    return MICRO_OK;
}

micro_status check_matrix(const micro_mx4_matrix* m) {
    if (!m) return refuse("a packed matrix is NULL");
    if (micro_status st = check_sides(m->rows, m->cols)) return st;
    if (m->rows > 0 && m->cols > 0 && (!m->codes || !m->scales)) return refuse("a packed matrix has NULL codes or scales");
    if (!aligned_to(m->codes, 16) || !aligned_to(m->scales, 4))
        return refuse("codes are not aligned to 16 bytes, or scales to 4");
    return MICRO_OK;
}

Mx4 matrix_of(const micro_mx4_matrix& m) {
    return {static_cast<char*>(m.codes), static_cast<uint8_t*>(m.scales), m.rows, m.cols, groups_of(m.cols)};
}
RowSpan codes_of(const micro_mx4_matrix* m) { return m ? run_of(m->codes, m->rows * groups_of(m->cols), kMxBytes) : RowSpan{}; }
RowSpan scales_of(const micro_mx4_matrix* m) { return m ? run_of(m->scales, m->rows * groups_of(m->cols), kMxBlocks) : RowSpan{}; }

micro_status check_values(const void* at, int32_t type, int64_t stride, int64_t rows, int64_t cols) {
    if (!type_valid(type)) return refuse("unknown type");
    if (micro_status st = check_sides(rows, cols)) return st;
    return check_strided(at, stride, rows, cols, type_bytes(type));
}
RowSpan values_of(const void* at, int32_t type, int64_t stride, int64_t rows, int64_t cols) {
    return {at, rows, stride * type_bytes(type), cols * type_bytes(type)};
}

micro_status check_product(const micro_mx4_matrix* a, const micro_mx4_matrix* b, const void* out, int32_t type,
                           int64_t stride) {
    if (micro_status st = check_matrix(a)) return st;
    if (micro_status st = check_matrix(b)) return st;
    if (a->cols != b->cols) return refuse("the matrices' rows differ in length");
    return check_values(out, type, stride, a->rows, b->rows);
}

Mx4Product product_of(const micro_mx4* mx, const micro_mx4_matrix* a, const micro_mx4_matrix* b, int32_t accumulate,
                      void* out, int32_t type, int64_t stride) {
    return {matrix_of(*a), matrix_of(*b), {out, stride, type}, accumulate != 0, mx->compute_units, mx->parts};
}

}  // namespace

extern "C" {

micro_status micro_mx4_bytes(int64_t rows, int64_t cols, int64_t* codes, int64_t* scales) {
    if (!codes || !scales) return refuse("an output is NULL");
    if (micro_status st = check_sides(rows, cols)) return st;
    *codes = rows * groups_of(cols) * kMxBytes;
    *scales = rows * groups_of(cols) * kMxBlocks;
    return MICRO_OK;
}

micro_status micro_mx4_init(micro_mx4** out, void* hip_stream) {
    if (!out) return refuse("mx is NULL");
    *out = nullptr;
    int device = -1, units = 0;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&units, hipDeviceAttributeMultiprocessorCount, device);
    if (e != hipSuccess) return report_hip(e, "device of the 4-bit calls");
    micro_mx4* mx = new (std::nothrow) micro_mx4;
    if (!mx) return MICRO_ENOMEM;
    mx->device = device;
    mx->compute_units = std::max(units, 8);
    mx->stream = static_cast<hipStream_t>(hip_stream);
    // with the handle, so that any of its calls may be captured into a graph
    if (micro_status st = ensure(&mx->memory, "4-bit products",
                                 [&](Parts& p) { p.take(mx->parts, mx->compute_units * kMxParts * 4); })) {
        delete mx;
        return st;
    }
    *out = mx;
    return MICRO_OK;
}

micro_status micro_mx4_pack(micro_mx4* mx, const void* x, int32_t type, int64_t stride, int64_t rows, int64_t cols,
                            const micro_mx4_matrix* packed, const micro_mx4_matrix* turned) {
    if (!mx) return refuse("mx is NULL");
    if (micro_status st = check_values(x, type, stride, rows, cols)) return st;
    if (!packed && !turned) return refuse("no output");
    if (packed) {
        if (micro_status st = check_matrix(packed)) return st;
        if (packed->rows != rows || packed->cols != cols) return refuse("packed is not rows x cols");
    }
    if (turned) {
        if (micro_status st = check_matrix(turned)) return st;
        if (turned->rows != cols || turned->cols != rows) return refuse("turned is not cols x rows");
    }
    const Region regions[] = {{values_of(x, type, stride, rows, cols), false}, {codes_of(packed), true},
                              {scales_of(packed), true}, {codes_of(turned), true}, {scales_of(turned), true}};
    if (micro_status st = check_apart(regions)) return st;
    CallDevice scope(mx->device);
    return report_hip(launch_mx4_pack({const_cast<void*>(x), stride, type}, rows, cols, packed ? matrix_of(*packed) : Mx4{},
                                      turned ? matrix_of(*turned) : Mx4{}, mx->stream),
                      "4-bit packing launch");
}

micro_status micro_mx4_unpack(micro_mx4* mx, const micro_mx4_matrix* packed, void* out, int32_t type, int64_t stride) {
    if (!mx) return refuse("mx is NULL");
    if (micro_status st = check_matrix(packed)) return st;
    if (micro_status st = check_values(out, type, stride, packed->rows, packed->cols)) return st;
    const Region regions[] = {{codes_of(packed), false}, {scales_of(packed), false},
                              {values_of(out, type, stride, packed->rows, packed->cols), true}};
    if (micro_status st = check_apart(regions)) return st;
    CallDevice scope(mx->device);
    return report_hip(launch_mx4_unpack(matrix_of(*packed), {out, stride, type}, mx->stream), "4-bit unpacking launch");
}

micro_status micro_mx4_product(micro_mx4* mx, const micro_mx4_matrix* a, const micro_mx4_matrix* b, int32_t accumulate,
                               void* out, int32_t type, int64_t stride) {
    if (!mx) return refuse("mx is NULL");
    if (micro_status st = check_product(a, b, out, type, stride)) return st;
    const Region regions[] = {{codes_of(a), false}, {scales_of(a), false}, {codes_of(b), false}, {scales_of(b), false},
                              {values_of(out, type, stride, a->rows, b->rows), true}};
    if (micro_status st = check_apart(regions)) return st;
    CallDevice scope(mx->device);
    return report_hip(launch_mx4_product(product_of(mx, a, b, accumulate, out, type, stride), mx->stream), "4-bit product launch");
}

micro_status micro_mx4_linear(micro_mx4* mx, const void* x, int32_t x_type, int64_t x_stride, const micro_mx4_matrix* a,
                              const micro_mx4_matrix* b, int32_t accumulate, void* out, int32_t type, int64_t stride) {
    if (!mx) return refuse("mx is NULL");
    if (micro_status st = check_product(a, b, out, type, stride)) return st;
    if (micro_status st = check_values(x, x_type, x_stride, a->rows, a->cols)) return st;
    const Region regions[] = {{codes_of(a), true}, {scales_of(a), true}, {codes_of(b), false}, {scales_of(b), false},
                              {values_of(x, x_type, x_stride, a->rows, a->cols), false},
                              {values_of(out, type, stride, a->rows, b->rows), true}};
    if (micro_status st = check_apart(regions)) return st;
    CallDevice scope(mx->device);
    return report_hip(launch_mx4_linear({const_cast<void*>(x), x_stride, x_type},
                                        product_of(mx, a, b, accumulate, out, type, stride), mx->stream),
                      "4-bit product launch");
}

void micro_mx4_free(micro_mx4* mx) {
    if (!mx) return;
    CallDevice scope(mx->device);
    (void)hipStreamSynchronize(mx->stream);
    if (mx->memory) (void)hipFree(mx->memory);
    delete mx;
}

}  // extern "C"

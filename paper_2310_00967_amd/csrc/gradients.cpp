// Host side of the gradient set's entry points (micro_grads_*).
#include <algorithm>
#include <cmath>
#include <new>
#include <utility>
#include <vector>

#include "gradients_kernel.h"
#include "host_util.h"
#include "micro_sparsify.h"

struct micro_grads {
    int device = -1;
    hipStream_t stream = nullptr;
    int64_t total = 0;                                    // values of all tensors
    std::vector<std::pair<const void*, int64_t>> ranges;  // address and bytes of every tensor that has any, by address
    void* scratch = nullptr;                              // partials, pieces
    micro::GradSetDevice dev{};
};

namespace {

using namespace micro;

// Values of a piece: a multiple of what a workgroup loads in one round.  Long
// sets take kPieceMax, whose 24-byte record is nothing beside its values;
// shorter ones as much less as gives every workgroup of a full grid a piece.
constexpr int64_t kPieceMax = 32768, kPieceMin = 4096;

int64_t piece_length(int64_t total) {
    int64_t piece = kPieceMax;
    while (piece > kPieceMin && total / piece < kGradGridMax) piece /= 2;
    return piece;
}

micro_status build(micro_grads* g, int32_t count, void* const* tensors, const int64_t* sizes, const int32_t* types) {
    const int64_t piece = piece_length(g->total);
    std::vector<GradPiece> pieces;
    int64_t offset = 0;
    for (int32_t i = 0; i < count; ++i) {
        const int64_t bytes = type_bytes(types[i]);
        for (int64_t at = 0; at < sizes[i]; at += piece)
            pieces.push_back({static_cast<char*>(tensors[i]) + at * bytes, offset + at,
                              static_cast<int32_t>(std::min(piece, sizes[i] - at)), types[i]});
        offset += sizes[i];
        if (sizes[i] > 0) g->ranges.emplace_back(tensors[i], sizes[i] * bytes);
    }
    std::sort(g->ranges.begin(), g->ranges.end());
    for (size_t i = 1; i < g->ranges.size(); ++i)
        if (share_bytes(g->ranges[i - 1].first, g->ranges[i - 1].second, g->ranges[i].first, g->ranges[i].second))
            return refuse("two tensors of the set share memory");
    hipError_t e = hipGetDevice(&g->device);
    if (e != hipSuccess) return report_hip(e, "hipGetDevice");
    const size_t head = kGradGridMax * sizeof(double);
    e = hipMalloc(&g->scratch, head + pieces.size() * sizeof(GradPiece));
    if (e != hipSuccess) {
        forget_hip_error();
        g->scratch = nullptr;
        set_thread_error("device scratch of a set of %lld values: %s", static_cast<long long>(g->total),
                         hipGetErrorString(e));
        return MICRO_ENOMEM;
    }
    g->dev.partials = static_cast<double*>(g->scratch);
    g->dev.pieces = reinterpret_cast<const GradPiece*>(static_cast<char*>(g->scratch) + head);
    g->dev.count = static_cast<int64_t>(pieces.size());
    g->dev.total = g->total;
    if (!pieces.empty())
        e = hipMemcpyAsync(const_cast<GradPiece*>(g->dev.pieces), pieces.data(), pieces.size() * sizeof(GradPiece),
                           hipMemcpyHostToDevice, g->stream);
    if (e == hipSuccess) e = hipStreamSynchronize(g->stream);  // the host's copy of the pieces ends here
    return report_hip(e, "upload of the gradient set");
}

void release(micro_grads* g) {
    if (!g) return;
    CallDevice scope(g->device);
    if (g->scratch) {
        (void)hipStreamSynchronize(g->stream);
        (void)hipFree(g->scratch);
    }
    delete g;
}

// Whether [p, p + bytes) shares memory with a tensor of the set.
bool touches_set(const micro_grads* g, const void* p, int64_t bytes) {
    auto it = std::upper_bound(g->ranges.begin(), g->ranges.end(), std::make_pair(p, INT64_MAX));
    if (it != g->ranges.end() && share_bytes(it->first, it->second, p, bytes)) return true;
    return it != g->ranges.begin() && share_bytes((it - 1)->first, (it - 1)->second, p, bytes);
}

micro_status check_scalars(const micro_grads* g, const double* sumsq, const float* norm) {
    if (!aligned_to(sumsq, 8) || !aligned_to(norm, 4)) return refuse("a scalar's address is not aligned");
    if ((sumsq && touches_set(g, sumsq, 8)) || (norm && touches_set(g, norm, 4)) ||
        (sumsq && norm && share_bytes(sumsq, 8, norm, 4)))
        return refuse("a scalar shares memory with the set or the other scalar");
    return MICRO_OK;
}

// The clipping's first pass unless the caller has the sum, and its second.
micro_status scale(micro_grads* g, double max_norm, const double* sumsq, float* flat, float* norm) {
    if (!(max_norm > 0.0)) return refuse("max_norm is not positive");
    if (micro_status st = check_scalars(g, sumsq, norm)) return st;
    CallDevice scope(g->device);
    const bool needed = norm || std::isfinite(max_norm);
    if (needed && !sumsq) {
        const hipError_t e = launch_grads_sums(g->dev, g->stream);
        if (e != hipSuccess) return report_hip(e, "gradient norm launch");
    }
    return report_hip(launch_grads_scale(g->dev, needed, sumsq, max_norm, flat, norm, g->stream),
                      "gradient scale launch");
}

}  // namespace

extern "C" {

micro_status micro_grads_init(micro_grads** out, int32_t count, void* const* tensors, const int64_t* sizes,
                              const int32_t* types, void* hip_stream) {
    if (!out) return refuse("grads is NULL");
    *out = nullptr;
    if (count < 0 || (count > 0 && (!tensors || !sizes || !types))) return refuse("invalid tensor list");
    int64_t total = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (!type_valid(types[i])) return refuse("unknown tensor type");
        if (sizes[i] < 0 || sizes[i] > (INT64_MAX >> 3) - total) return refuse("invalid tensor size");
        if (sizes[i] > 0 && (!tensors[i] || !aligned_to(tensors[i], type_bytes(types[i]))))
            return refuse("a tensor's address is NULL or not aligned to its type");
        total += sizes[i];
    }
    micro_grads* g = new (std::nothrow) micro_grads;
    if (!g) return MICRO_ENOMEM;
    g->stream = static_cast<hipStream_t>(hip_stream);
    g->total = total;
    micro_status st;
    try {
        st = build(g, count, tensors, sizes, types);
    } catch (const std::bad_alloc&) {
        set_thread_error("host memory of the gradient set");
        st = MICRO_ENOMEM;
    }
    if (st != MICRO_OK) {
        release(g);
        return st;
    }
    *out = g;
    return MICRO_OK;
}

micro_status micro_grads_norm(micro_grads* g, double* sumsq, float* norm) {
    if (!g) return refuse("grads is NULL");
    if (!sumsq && !norm) return refuse("NULL outputs");
    if (micro_status st = check_scalars(g, sumsq, norm)) return st;
    CallDevice scope(g->device);
    return report_hip(launch_grads_norm(g->dev, sumsq, norm, g->stream), "gradient norm launch");
}

micro_status micro_grads_clip(micro_grads* g, double max_norm, const double* sumsq, float* norm) {
    if (!g) return refuse("grads is NULL");
    return scale(g, max_norm, sumsq, nullptr, norm);
}

micro_status micro_grads_flatten(micro_grads* g, double max_norm, const double* sumsq, float* flat, float* norm) {
    if (!g) return refuse("grads is NULL");
    const int64_t bytes = g->total * 4;
    if (bytes > 0 && (!flat || !aligned_to(flat, 4))) return refuse("flat is NULL or not 4-byte aligned");
    for (const auto& r : g->ranges)
        if (share_bytes(r.first, r.second, flat, bytes)) return refuse("flat shares memory with a tensor of the set");
    if (share_bytes(sumsq, sumsq ? 8 : 0, flat, bytes) || share_bytes(norm, norm ? 4 : 0, flat, bytes))
        return refuse("flat shares memory with a scalar");
    if (bytes == 0) return micro_grads_clip(g, max_norm, sumsq, norm);
    return scale(g, max_norm, sumsq, flat, norm);
}

void micro_grads_free(micro_grads* g) { release(g); }

}  // extern "C"

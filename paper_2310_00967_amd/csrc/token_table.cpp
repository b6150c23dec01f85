// Host side of the token table's entry points (micro_table_*).
#include <algorithm>
#include <cmath>
#include <new>

#include "host_util.h"
#include "lookup_kernel.h"
#include "loss_kernel.h"
#include "micro_sparsify.h"
#include "strided_rows.h"

namespace {

using namespace micro;

constexpr int64_t kMostTokens = int64_t(1) << 22;
// Of the loss: 32-bit offsets within a product tile.
constexpr int64_t kMostLossVocab = int64_t(1) << 22;
constexpr int64_t kMostDim = 65536;

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

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

}  // namespace

struct micro_table {
    int device = -1;
    int compute_units = 256;
    hipStream_t stream = nullptr;
    int64_t vocab = 0, max_tokens = 0;
    int32_t dim = 0, type = 0;
    micro_table_config cfg{};
    // scratch, allocated by the first call that needs it
    void* lookup_memory = nullptr;
    LookupGradScratch lookup{};
    void* loss_memory = nullptr;       // of the loss
    void* table_memory = nullptr;      // the table's padded copy
    void* gradient_memory = nullptr;   // of its gradients
    LossCall loss{};                   // the scratch members are set

    int64_t size() const { return type_bytes(type); }
};

namespace {

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

void release(micro_table* t) {
    if (!t) return;
    CallDevice scope(t->device);
    if (t->device >= 0) (void)hipStreamSynchronize(t->stream);
    for (void* p : {t->lookup_memory, t->loss_memory, t->table_memory, t->gradient_memory})
        if (p) (void)hipFree(p);
    delete t;
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

// An argument's rows, and `values` values one after the other, in bytes.
RowSpan rows_of(const micro_table* t, const void* at, int64_t rows, int64_t stride) {
    return {at, rows, stride * t->size(), t->dim * t->size()};
}
RowSpan run_of(const void* at, int64_t values, int64_t size) { return {at, 1, values * size, values * size}; }

micro_status check_rows(const micro_table* t, const void* at, int64_t stride, int64_t rows) {
    if (stride < t->dim) return refuse("a row stride is below the table's dim");
    if (stride > (int64_t(1) << 32) || rows > (int64_t(1) << 56) / stride)
        return refuse("a row stride is above 2^32, or the rows end past 2^56 values");
    if (rows > 0 && (!at || !aligned_to(at, t->size()))) return refuse("rows are NULL or not aligned to their type");
    return MICRO_OK;
}

micro_status check_tokens(const micro_table* t, const void* ids, int32_t ids_type, int64_t tokens) {
    if (tokens < 0) return refuse("a negative number of tokens");
    if (tokens > t->max_tokens) {
        set_thread_error("%lld tokens, and the handle holds %lld", static_cast<long long>(tokens),
                         static_cast<long long>(t->max_tokens));
        return MICRO_ECAPACITY;
    }
    if (ids_type != MICRO_IDS_I32 && ids_type != MICRO_IDS_I64) return refuse("unknown type of ids");
    if (tokens > 0 && (!ids || !aligned_to(ids, ids_type == MICRO_IDS_I64 ? 8 : 4)))
        return refuse("ids are NULL or not aligned to their type");
    return MICRO_OK;
}

RowSpan ids_of(const void* ids, int32_t ids_type, int64_t tokens) {
    return run_of(ids, tokens, ids_type == MICRO_IDS_I64 ? 8 : 4);
}

// The loss's scratch for the handle's largest call.
micro_status loss_scratch(micro_table* t, bool copy_table, bool gradients) {
    LossCall& c = t->loss;
    const int64_t dim = round_up(t->dim, kProductDepth), vocab = round_up(t->vocab, kProductDepth);
    const int64_t tokens = round_up(std::max<int64_t>(t->max_tokens, 1), kProductDepth);
    const bool split = t->type == MICRO_TYPE_F32;
    const int64_t planes = split ? kSplitPlanes : 1;
    // a token block: as many tokens as the scores' scratch holds
    const int64_t score = split ? 4 + 2 * kSplitPlanes : 2;
    const int64_t fits = std::max<int64_t>(t->cfg.score_bytes / (vocab * score) / 256, 1) * 256;
    c.block = std::min(fits, round_up(tokens, 256));
    // [granule][block]; shorter calls have more granules and shorter blocks
    const int64_t granules = std::max({round_up(t->vocab, 256) / kGranule * c.block,
                                       round_up(t->vocab, 256) / kGranuleSome * kSomeTokens,
                                       round_up(t->vocab, 256) / kGranuleFew * kFewTokens});
    if (micro_status st = ensure(&t->loss_memory, "token loss", [&](Parts& p) {
            p.take(c.count, 12);
            p.take(c.chunks, tokens * 4 / 1024 + 4);
            p.take(c.rows, tokens * 4);
            p.take(c.labels, tokens * 4);
            p.take(c.counted_losses, tokens * 4);
            p.take(c.label_logit, c.block * 4);
            p.take(c.label_rest, c.block * 4);
            p.take(c.softmax, c.block * 8);
            p.take(c.stats, granules * 8);
            p.take(c.h, planes * tokens * dim * 2);
            p.take(c.parts, 2 * t->compute_units * kPartTile * 4);
        }))
        return st;
    if (copy_table)
        if (micro_status st = ensure(&t->table_memory, "token loss's copy of the table",
                                     [&](Parts& p) { p.take(c.w, planes * t->vocab * dim * 2); }))
            return st;
    if (!gradients) return MICRO_OK;
    return ensure(&t->gradient_memory, "token loss's gradients", [&](Parts& p) {
        p.take(c.scores, c.block * vocab * (split ? 4 : 2));
        if (split) p.take(c.split, planes * c.block * vocab * 2);
        p.take(c.partials, 2 * t->compute_units * kWideTile * 4);
        if (t->max_tokens > c.block)
            p.take(c.carried, round_up(t->vocab, 256) * round_up(t->dim, 256) * 4);
    });
}

micro_status run_loss(micro_table* t, const void* hidden, int64_t hidden_stride, const void* weight, int64_t weight_stride,
                      const void* targets, int32_t targets_type, int64_t tokens, bool mean, float* losses, float* loss,
                      bool gradients, double scale, bool accumulate, void* dhidden, int64_t dhidden_stride,
                      void* dweight, int64_t dweight_stride) {
    if (!t) return refuse("table is NULL");
    if (micro_status st = check_tokens(t, targets, targets_type, tokens)) return st;
    if (micro_status st = check_rows(t, hidden, hidden_stride, tokens)) return st;
    if (micro_status st = check_rows(t, weight, weight_stride, t->vocab)) return st;
    if (!loss || !aligned_to(loss, 4) || (tokens > 0 && !losses) || !aligned_to(losses, 4))
        return refuse("loss or losses is NULL or not 4-byte aligned");
    if (gradients) {
        if (micro_status st = check_rows(t, dhidden, dhidden_stride, tokens)) return st;
        if (micro_status st = check_rows(t, dweight, dweight_stride, t->vocab)) return st;
        if (!std::isfinite(scale) || !std::isfinite(static_cast<float>(scale))) return refuse("scale is not finite");
    }
    if (t->vocab > kMostLossVocab) {
        set_thread_error("a loss over %lld rows: at most 2^22", static_cast<long long>(t->vocab));
        return MICRO_ERANGE;
    }
    const Region regions[] = {
        {rows_of(t, hidden, tokens, hidden_stride), false},
        {rows_of(t, weight, t->vocab, weight_stride), false},
        {ids_of(targets, targets_type, tokens), false},
        {run_of(losses, tokens, 4), true},
        {run_of(loss, 1, 4), true},
        {rows_of(t, dhidden, gradients ? tokens : 0, dhidden_stride), true},
        {rows_of(t, dweight, gradients ? t->vocab : 0, dweight_stride), true},
    };
    if (micro_status st = check_apart(regions)) return st;
    CallDevice scope(t->device);
    LossCall c{};
    c.type = t->type;
    c.dim = t->dim;
    c.table = {const_cast<void*>(weight), weight_stride, t->type};
    if (micro_status st = loss_scratch(t, !table_in_place(c), gradients)) return st;
    c = t->loss;
    c.type = t->type;
    c.vocab = t->vocab;
    c.vocab_padded = round_up(t->vocab, kProductDepth);
    c.dim = t->dim;
    c.dim_padded = static_cast<int32_t>(round_up(t->dim, kProductDepth));
    c.tokens = tokens;
    c.hidden = {const_cast<void*>(hidden), hidden_stride, t->type};
    c.table = {const_cast<void*>(weight), weight_stride, t->type};
    c.targets = {targets, targets_type == MICRO_IDS_I64};
    c.ignored = t->cfg.ignored;
    c.mean = mean;
    c.scale = static_cast<float>(scale);
    c.losses = losses;
    c.loss = loss;
    c.gradients = gradients;
    c.accumulate = accumulate;
    c.dhidden = {dhidden, dhidden_stride, t->type};
    c.dtable = {dweight, dweight_stride, t->type};
    c.compute_units = t->compute_units;
    return report_hip(launch_loss(c, t->stream), "token loss launch");
}

}  // namespace

extern "C" {

void micro_table_config_default(micro_table_config* cfg) {
    if (cfg) *cfg = {-1, -100, int64_t(1) << 31};
}

micro_status micro_table_init(micro_table** out, int64_t vocab, int32_t dim, int64_t max_tokens, int32_t type,
                              void* hip_stream, const micro_table_config* cfg) {
    if (!out) return refuse("table is NULL");
    *out = nullptr;
    if (vocab < 1 || dim < 1 || max_tokens < 0 || !type_valid(type)) return refuse("invalid table sizes or type");
    if (vocab > INT32_MAX - 1 || dim > kMostDim || max_tokens > kMostTokens) {
        set_thread_error("a table of %lld x %d with %lld tokens: at most 2^31 - 2 x 65536 and 2^22",
                         static_cast<long long>(vocab), dim, static_cast<long long>(max_tokens));
        return MICRO_ERANGE;
    }
    if (cfg && cfg->score_bytes < 0) return refuse("score_bytes is negative");
    int device = -1, units = 0;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&units, hipDeviceAttributeMultiprocessorCount, device);
    if (e != hipSuccess) return report_hip(e, "device of the token table");
    micro_table* t = new (std::nothrow) micro_table;
    if (!t) return MICRO_ENOMEM;
    t->device = device;
    t->compute_units = std::max(units, 8);
    t->stream = static_cast<hipStream_t>(hip_stream);
    t->vocab = vocab;
    t->dim = dim;
    t->max_tokens = max_tokens;
    t->type = type;
    if (cfg)
        t->cfg = *cfg;
    else
        micro_table_config_default(&t->cfg);
    *out = t;
    return MICRO_OK;
}

micro_status micro_table_lookup(micro_table* t, const void* weight, int64_t weight_stride, const void* ids,
                                int32_t ids_type, int64_t tokens, double scale, void* out, int64_t out_stride) {
    if (!t) return refuse("table is NULL");
    if (micro_status st = check_tokens(t, ids, ids_type, tokens)) return st;
    if (micro_status st = check_rows(t, weight, weight_stride, t->vocab)) return st;
    if (micro_status st = check_rows(t, out, out_stride, tokens)) return st;
    const Region regions[] = {{rows_of(t, weight, t->vocab, weight_stride), false},
                              {ids_of(ids, ids_type, tokens), false},
                              {rows_of(t, out, tokens, out_stride), true}};
    if (micro_status st = check_apart(regions)) return st;
    CallDevice scope(t->device);
    return report_hip(launch_lookup({const_cast<void*>(weight), weight_stride, t->type}, t->vocab, t->dim,
                                    {ids, ids_type == MICRO_IDS_I64}, tokens, static_cast<float>(scale),
                                    {out, out_stride, t->type}, t->stream),
                      "token lookup launch");
}

micro_status micro_table_lookup_grad(micro_table* t, const void* grad, int64_t grad_stride, const void* ids,
                                     int32_t ids_type, int64_t tokens, double scale, int32_t accumulate, void* dweight,
                                     int64_t dweight_stride) {
    if (!t) return refuse("table is NULL");
    if (micro_status st = check_tokens(t, ids, ids_type, tokens)) return st;
    if (micro_status st = check_rows(t, grad, grad_stride, tokens)) return st;
    if (micro_status st = check_rows(t, dweight, dweight_stride, t->vocab)) return st;
    const Region regions[] = {{rows_of(t, grad, tokens, grad_stride), false},
                              {ids_of(ids, ids_type, tokens), false},
                              {rows_of(t, dweight, t->vocab, dweight_stride), true}};
    if (micro_status st = check_apart(regions)) return st;
    CallDevice scope(t->device);
    LookupGradScratch& s = t->lookup;
    const int64_t words = t->max_tokens * 4;
    if (micro_status st = ensure(&t->lookup_memory, "token lookup's gradient", [&](Parts& p) {
            p.take(s.keys[0], words);
            p.take(s.keys[1], words);
            p.take(s.order[0], words);
            p.take(s.order[1], words);
            p.take(s.partials, round_up(t->max_tokens, kSumChunk) / kSumChunk * 2 * t->dim * 4);
        }))
        return st;
    return report_hip(launch_lookup_grad({const_cast<void*>(grad), grad_stride, t->type}, tokens,
                                         {ids, ids_type == MICRO_IDS_I64}, t->cfg.padding_id,
                                         static_cast<float>(scale), accumulate != 0,
                                         {dweight, dweight_stride, t->type}, t->vocab, t->dim, s, t->stream),
                      "token lookup gradient launch");
}

micro_status micro_table_loss(micro_table* t, const void* hidden, int64_t hidden_stride, const void* weight,
                              int64_t weight_stride, const void* targets, int32_t targets_type, int64_t tokens,
                              int32_t mean, float* losses, float* loss) {
    return run_loss(t, hidden, hidden_stride, weight, weight_stride, targets, targets_type, tokens, mean != 0, losses,
                    loss, false, 1.0, false, nullptr, 0, nullptr, 0);
}

micro_status micro_table_loss_grad(micro_table* t, const void* hidden, int64_t hidden_stride, const void* weight,
                                   int64_t weight_stride, const void* targets, int32_t targets_type, int64_t tokens,
                                   int32_t mean, double scale, int32_t accumulate, float* losses, float* loss,
                                   void* dhidden, int64_t dhidden_stride, void* dweight, int64_t dweight_stride) {
    return run_loss(t, hidden, hidden_stride, weight, weight_stride, targets, targets_type, tokens, mean != 0, losses,
                    loss, true, scale, accumulate != 0, dhidden, dhidden_stride, dweight, dweight_stride);
}

void micro_table_free(micro_table* t) { release(t); }

}  // extern "C"

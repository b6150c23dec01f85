// Marshalling of the Python binding's calls on a context (Caller.step, .ef_step
// and .sweep), on a token table (TableCaller.lookup and .sample) and on 4-bit matrices
// (MxCaller): they check the tensors, call the C ABI of include/micro_sparsify.h and wrap
// the results.  They take the plain case
// only (exact torch.Tensor buffers, Python floats and ints, every check
// passed) and return None otherwise, with nothing called: the Python methods
// then go their own way, which names what is wrong.  A nonzero status comes
// back as that int.  The C functions run without the interpreter lock, as
// ctypes runs them.
//
// In Python a step's checks, conversions and two views took 4.5 us of a call
// whose launch and wait take 12.
#include <Python.h>

#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>
#include <torch/torch.h>

#include <cstdint>

#include "micro_sparsify.h"

namespace {

struct Caller {
    PyObject_HEAD
    decltype(&micro_sparsify_step) step;
    decltype(&micro_ef_step) ef_step;
    decltype(&micro_sweep_step) sweep;
    micro_ctx* ctx;
    int64_t n_total;
    int device;
};

constexpr int kMaxSweepWorld = 64;

// The tensor of a plain 1-D contiguous buffer of the wanted type on the
// context's device with at least `least` values (exactly that many for
// `exact`), or null.
const at::Tensor* buffer(PyObject* o, const Caller* c, at::ScalarType type, int64_t least, bool exact) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.layout() != at::kStrided || t.scalar_type() != type || !t.is_cuda() || t.get_device() != c->device ||
        !t.is_contiguous())
        return nullptr;
    if (exact ? t.numel() != least : (t.dim() != 1 || t.numel() < least)) return nullptr;
    return &t;
}

bool integer(PyObject* o, int64_t* v) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &over);
    return over == 0;
}

bool real(PyObject* o, double* v) {
    if (!PyFloat_CheckExact(o)) return false;
    *v = PyFloat_AS_DOUBLE(o);
    return true;
}

struct Buffers {
    const at::Tensor *grad, *residual, *idx, *val;
};

bool buffers(const Caller* c, PyObject* grad, PyObject* residual, PyObject* idx, PyObject* val, int64_t capacity,
             Buffers* b) {
    b->grad = buffer(grad, c, at::kFloat, c->n_total, true);
    b->residual = buffer(residual, c, at::kFloat, c->n_total, true);
    b->idx = buffer(idx, c, at::kInt, capacity, false);
    b->val = buffer(val, c, at::kFloat, capacity, false);
    return b->grad && b->residual && b->idx && b->val;
}

int64_t partition_length(int64_t n, int64_t rank, int64_t world) {
    return (rank + 1) * n / world - rank * n / world;
}

// Views of the first k pairs, or false with the Python error set.
struct Pairs {
    THPObjectPtr idx, val;
    bool make(const Buffers& b, int64_t k) {
        idx = THPVariable_Wrap(b.idx->slice(0, 0, k));
        if (!idx.get()) return false;
        val = THPVariable_Wrap(b.val->slice(0, 0, k));
        return val.get() != nullptr;
    }
};

// A list of n new objects from make(i), or null with the Python error set.
template <class Make>
PyObject* list_of(int64_t n, Make make) {
    THPObjectPtr list(PyList_New(n));
    if (!list.get()) return nullptr;
    for (int64_t i = 0; i < n; ++i) {
        PyObject* item = make(i);
        if (!item) return nullptr;
        PyList_SET_ITEM(list.get(), i, item);
    }
    return list.release();
}

// step(grad, residual, rank, world, density, theta, out_idx, out_val)
PyObject* caller_step(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    Caller* c = reinterpret_cast<Caller*>(self);
    int64_t rank, world;
    double density, theta;
    Buffers b;
    HANDLE_TH_ERRORS
    if (n != 8 || !integer(args[2], &rank) || !integer(args[3], &world) || world < 1 || world > INT32_MAX ||
        rank < 0 || rank >= world || !real(args[4], &density) || !real(args[5], &theta) ||
        !buffers(c, args[0], args[1], args[6], args[7], partition_length(c->n_total, rank, world), &b))
        Py_RETURN_NONE;
    const float* grad = static_cast<const float*>(b.grad->data_ptr());
    float* residual = static_cast<float*>(b.residual->data_ptr());
    int32_t* idx = static_cast<int32_t*>(b.idx->data_ptr());
    float* val = static_cast<float*>(b.val->data_ptr());
    int64_t k = 0;
    micro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = c->step(c->ctx, grad, residual, static_cast<int32_t>(rank), static_cast<int32_t>(world), density, &theta,
                 idx, val, &k);
    Py_END_ALLOW_THREADS
    if (st != MICRO_OK) return PyLong_FromLong(st);
    Pairs p;
    if (!p.make(b, k)) return nullptr;
    return Py_BuildValue("(LdOO)", static_cast<long long>(k), theta, p.idx.get(), p.val.get());
    END_HANDLE_TH_ERRORS
}

// ef_step(grad, residual, t, worker, world, density, theta, out_idx, out_val, local_error)
PyObject* caller_ef_step(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    Caller* c = reinterpret_cast<Caller*>(self);
    int64_t t, worker, world;
    double density, theta, sumsq = 0.0;
    Buffers b;
    HANDLE_TH_ERRORS
    if (n != 10 || !integer(args[2], &t) || !integer(args[3], &worker) || !integer(args[4], &world) || t < 0 ||
        world < 1 || world > INT32_MAX || worker < 0 || worker >= world || !real(args[5], &density) ||
        !real(args[6], &theta) || !PyBool_Check(args[9]))
        Py_RETURN_NONE;
    const int64_t part = (t % world + worker) % world;
    if (!buffers(c, args[0], args[1], args[7], args[8], partition_length(c->n_total, part, world), &b))
        Py_RETURN_NONE;
    const float* grad = static_cast<const float*>(b.grad->data_ptr());
    float* residual = static_cast<float*>(b.residual->data_ptr());
    int32_t* idx = static_cast<int32_t*>(b.idx->data_ptr());
    float* val = static_cast<float*>(b.val->data_ptr());
    const bool error = args[9] == Py_True;
    int64_t k = 0;
    int32_t cycle = 0;
    micro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = c->ef_step(c->ctx, grad, residual, t, static_cast<int32_t>(worker), static_cast<int32_t>(world), density,
                    &theta, idx, val, &k, &cycle, error ? &sumsq : nullptr);
    Py_END_ALLOW_THREADS
    if (st != MICRO_OK) return PyLong_FromLong(st);
    Pairs p;
    if (!p.make(b, k)) return nullptr;
    if (error)
        return Py_BuildValue("(LdiOOd)", static_cast<long long>(k), theta, cycle, p.idx.get(), p.val.get(), sumsq);
    return Py_BuildValue("(LdiOO)", static_cast<long long>(k), theta, cycle, p.idx.get(), p.val.get());
    END_HANDLE_TH_ERRORS
}

// sweep(grad, residual, world, density, thetas, out_idx, out_val, want_sumsq)
PyObject* caller_sweep(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    Caller* c = reinterpret_cast<Caller*>(self);
    int64_t world, k[kMaxSweepWorld], total = 0;
    double density, theta[kMaxSweepWorld], sumsq[kMaxSweepWorld];
    Buffers b;
    HANDLE_TH_ERRORS
    if (n != 8 || !integer(args[2], &world) || world < 1 || world > kMaxSweepWorld || !real(args[3], &density) ||
        !PyList_CheckExact(args[4]) || PyList_GET_SIZE(args[4]) != world || !PyBool_Check(args[7]))
        Py_RETURN_NONE;
    for (int64_t r = 0; r < world; ++r)
        if (!real(PyList_GET_ITEM(args[4], r), &theta[r])) Py_RETURN_NONE;
    if (!buffers(c, args[0], args[1], args[5], args[6], c->n_total, &b)) Py_RETURN_NONE;
    const float* grad = static_cast<const float*>(b.grad->data_ptr());
    float* residual = static_cast<float*>(b.residual->data_ptr());
    int32_t* idx = static_cast<int32_t*>(b.idx->data_ptr());
    float* val = static_cast<float*>(b.val->data_ptr());
    const bool error = args[7] == Py_True;
    micro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = c->sweep(c->ctx, grad, residual, static_cast<int32_t>(world), density, theta, idx, val, k,
                  error ? sumsq : nullptr);
    Py_END_ALLOW_THREADS
    if (st != MICRO_OK) return PyLong_FromLong(st);
    for (int64_t r = 0; r < world; ++r) total += k[r];
    THPObjectPtr ks(list_of(world, [&](int64_t r) { return PyLong_FromLongLong(k[r]); }));
    if (!ks.get()) return nullptr;
    THPObjectPtr ths(list_of(world, [&](int64_t r) { return PyFloat_FromDouble(theta[r]); }));
    if (!ths.get()) return nullptr;
    THPObjectPtr sqs(error ? list_of(world, [&](int64_t r) { return PyFloat_FromDouble(sumsq[r]); })
                           : Py_NewRef(Py_None));
    if (!sqs.get()) return nullptr;
    Pairs p;
    if (!p.make(b, total)) return nullptr;
    return Py_BuildValue("(OOOOO)", ks.get(), ths.get(), sqs.get(), p.idx.get(), p.val.get());
    END_HANDLE_TH_ERRORS
}

// Caller(step, ef_step, sweep, ctx, n_total, device): the C functions' and the
// context's addresses, the vector's length and the device's index.
PyObject* caller_new(PyTypeObject* type, PyObject* args, PyObject*) {
    unsigned long long step, ef_step, sweep, ctx;
    long long n_total;
    int device;
    if (!PyArg_ParseTuple(args, "KKKKLi", &step, &ef_step, &sweep, &ctx, &n_total, &device)) return nullptr;
    Caller* c = reinterpret_cast<Caller*>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    c->step = reinterpret_cast<decltype(c->step)>(step);
    c->ef_step = reinterpret_cast<decltype(c->ef_step)>(ef_step);
    c->sweep = reinterpret_cast<decltype(c->sweep)>(sweep);
    c->ctx = reinterpret_cast<micro_ctx*>(ctx);
    c->n_total = n_total;
    c->device = device;
    return reinterpret_cast<PyObject*>(c);
}

// TableCaller: the lookup of a token table's rows, whose kernel takes 2 us, and the draw of
// tokens in the plain case: contiguous tensors, called on the handle's stream, with outputs
// of their own.  (In Python the lookup's checks, the allocation and the call took 9 us.)
struct TableCaller {
    PyObject_HEAD
    decltype(&micro_table_lookup) lookup;
    decltype(&micro_table_sample) sample;
    micro_table* table;
    int64_t vocab, dim;
    at::ScalarType type;
    int device;
    int64_t stream;  // c10's id of the handle's stream
};

// Neither requires its gradient nor carries a tangent.
bool outside_autograd(const at::Tensor& t) { return !t.requires_grad() && !t._fw_grad(/*level=*/0).defined(); }

// lookup(weight, ids, scale): the rows; None: not the plain case; an int: the
// call's status.
PyObject* table_lookup(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    TableCaller* c = reinterpret_cast<TableCaller*>(self);
    double scale;
    HANDLE_TH_ERRORS
    if (n != 3 || !THPVariable_CheckExact(args[0]) || !THPVariable_CheckExact(args[1]) || !real(args[2], &scale))
        Py_RETURN_NONE;
    const at::Tensor& weight = THPVariable_Unpack(args[0]);
    const at::Tensor& ids = THPVariable_Unpack(args[1]);
    const auto plain = [&](const at::Tensor& t) {
        return t.layout() == at::kStrided && t.is_cuda() && t.get_device() == c->device && t.is_contiguous() &&
               outside_autograd(t);
    };
    const bool wide = ids.scalar_type() == at::kLong;
    if (!plain(weight) || !plain(ids) || weight.scalar_type() != c->type || weight.dim() != 2 ||
        weight.size(0) != c->vocab || weight.size(1) != c->dim || (!wide && ids.scalar_type() != at::kInt))
        Py_RETURN_NONE;
    const c10::Device device(c10::DeviceType::CUDA, static_cast<c10::DeviceIndex>(c->device));
    if (c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getStream(device).id() != c->stream) Py_RETURN_NONE;
    c10::SmallVector<int64_t, 6> shape(ids.sizes().begin(), ids.sizes().end());
    shape.push_back(c->dim);
    at::Tensor out = at::empty(shape, weight.options());
    const void* from = weight.data_ptr();
    const void* at = ids.data_ptr();
    void* to = out.data_ptr();
    const int64_t tokens = ids.numel();
    micro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = c->lookup(c->table, from, c->dim, at, wide ? MICRO_IDS_I64 : MICRO_IDS_I32, tokens, scale, to, c->dim);
    Py_END_ALLOW_THREADS
    if (st != MICRO_OK) return PyLong_FromLong(st);
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// A number, or a tensor of one value a row, as one of sample's settings.
template <class Number>
bool setting(PyObject* from, int device, int64_t rows, at::ScalarType type, Number* number, const void** array) {
    if (THPVariable_CheckExact(from)) {
        const at::Tensor& t = THPVariable_Unpack(from);
        if (!t.is_cuda() || t.get_device() != device || !t.is_contiguous() || t.scalar_type() != type || t.numel() != rows ||
            !outside_autograd(t))
            return false;
        *array = t.data_ptr();
        return true;
    }
    if constexpr (std::is_same<Number, double>::value) {
        if (!PyLong_CheckExact(from)) return real(from, number);
        *number = PyLong_AsDouble(from);
        if (!PyErr_Occurred()) return true;
        PyErr_Clear();  // too large for one
        return false;
    }
    if (!PyLong_CheckExact(from)) return false;
    int overflow = 0;
    *number = PyLong_AsLongLongAndOverflow(from, &overflow);
    return overflow == 0;
}

// sample(logits, uniforms, temperature, top_k, top_p, min_p): (ids, logprobs); None and an
// int as above.
PyObject* table_sample(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    TableCaller* c = reinterpret_cast<TableCaller*>(self);
    HANDLE_TH_ERRORS
    if (n != 6 || !THPVariable_CheckExact(args[0]) || !THPVariable_CheckExact(args[1])) Py_RETURN_NONE;
    const at::Tensor& logits = THPVariable_Unpack(args[0]);
    const at::Tensor& uniforms = THPVariable_Unpack(args[1]);
    const auto plain = [&](const at::Tensor& t) {
        return t.layout() == at::kStrided && t.is_cuda() && t.get_device() == c->device && t.is_contiguous() &&
               outside_autograd(t);
    };
    const int64_t rows = uniforms.numel();
    const auto kind = logits.scalar_type();
    const int32_t type = kind == at::kFloat ? MICRO_TYPE_F32 : kind == at::kHalf ? MICRO_TYPE_F16
                         : kind == at::kBFloat16 ? MICRO_TYPE_BF16 : -1;
    if (!plain(logits) || !plain(uniforms) || type < 0 || uniforms.scalar_type() != at::kFloat || logits.dim() < 1 ||
        logits.size(-1) != c->vocab || logits.numel() != rows * c->vocab)
        Py_RETURN_NONE;
    micro_sampling s{};
    const void *temperatures = nullptr, *top_ks = nullptr, *top_ps = nullptr, *min_ps = nullptr;
    if (!setting(args[2], c->device, rows, at::kFloat, &s.temperature, &temperatures) ||
        !setting(args[3], c->device, rows, at::kInt, &s.top_k, &top_ks) ||
        !setting(args[4], c->device, rows, at::kFloat, &s.top_p, &top_ps) ||
        !setting(args[5], c->device, rows, at::kFloat, &s.min_p, &min_ps))
        Py_RETURN_NONE;
    s.temperatures = static_cast<const float*>(temperatures);
    s.top_ks = static_cast<const int32_t*>(top_ks);
    s.top_ps = static_cast<const float*>(top_ps);
    s.min_ps = static_cast<const float*>(min_ps);
    const c10::Device device(c10::DeviceType::CUDA, static_cast<c10::DeviceIndex>(c->device));
    if (c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getStream(device).id() != c->stream) Py_RETURN_NONE;
    at::Tensor ids = at::empty(uniforms.sizes(), uniforms.options().dtype(at::kLong));
    at::Tensor logprobs = at::empty(uniforms.sizes(), uniforms.options());
    const void* from = logits.data_ptr();
    const float* u = static_cast<const float*>(uniforms.data_ptr());
    void* to = ids.data_ptr();
    float* p = static_cast<float*>(logprobs.data_ptr());
    micro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = c->sample(c->table, from, type, c->vocab, rows, u, &s, to, MICRO_IDS_I64, p);
    Py_END_ALLOW_THREADS
    if (st != MICRO_OK) return PyLong_FromLong(st);
    THPObjectPtr first(THPVariable_Wrap(std::move(ids)));
    if (!first.get()) return nullptr;
    THPObjectPtr second(THPVariable_Wrap(std::move(logprobs)));
    if (!second.get()) return nullptr;
    return PyTuple_Pack(2, first.get(), second.get());
    END_HANDLE_TH_ERRORS
}

// TableCaller(lookup, sample, table, vocab, dim, type, device, stream): type is a
// MICRO_TYPE_*.
PyObject* table_caller_new(PyTypeObject* type, PyObject* args, PyObject*) {
    unsigned long long lookup, sample, table;
    long long vocab, dim, stream;
    int value_type, device;
    if (!PyArg_ParseTuple(args, "KKKLLiiL", &lookup, &sample, &table, &vocab, &dim, &value_type, &device, &stream)) return nullptr;
    TableCaller* c = reinterpret_cast<TableCaller*>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    c->lookup = reinterpret_cast<decltype(c->lookup)>(lookup);
    c->sample = reinterpret_cast<decltype(c->sample)>(sample);
    c->table = reinterpret_cast<micro_table*>(table);
    c->vocab = vocab;
    c->dim = dim;
    c->type = value_type == MICRO_TYPE_F32 ? at::kFloat : value_type == MICRO_TYPE_F16 ? at::kHalf : at::kBFloat16;
    c->device = device;
    c->stream = stream;
    return reinterpret_cast<PyObject*>(c);
}

PyMethodDef table_methods[] = {
    {"lookup", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(table_lookup)), METH_FASTCALL, nullptr},
    {"sample", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(table_sample)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject table_caller_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

// ---------------------------------------------------------------------------
// MxCaller: the 4-bit calls in the plain case: contiguous tensors on the device, called
// on the handle's stream, with outputs of their own.
struct MxCaller {
    PyObject_HEAD
    decltype(&micro_mx4_pack) pack;
    decltype(&micro_mx4_unpack) unpack;
    decltype(&micro_mx4_product) product;
    decltype(&micro_mx4_linear) linear;
    micro_mx4* mx;
    int device;
    int64_t stream;  // c10's id of the handle's stream
};

constexpr int64_t kGroup = 128, kGroupBytes = 64, kGroupBlocks = 4;

int32_t type_of(at::ScalarType t) {
    return t == at::kFloat ? MICRO_TYPE_F32 : t == at::kHalf ? MICRO_TYPE_F16 : t == at::kBFloat16 ? MICRO_TYPE_BF16 : -1;
}

bool plain_values(const at::Tensor& t, int device) {
    return t.layout() == at::kStrided && t.is_cuda() && t.get_device() == device && t.is_contiguous() && t.dim() >= 1 &&
           t.size(-1) > 0 && t.numel() > 0 && outside_autograd(t) && type_of(t.scalar_type()) >= 0;
}

bool on_stream(int device, int64_t stream) {
    const c10::Device d(c10::DeviceType::CUDA, static_cast<c10::DeviceIndex>(device));
    return c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getStream(d).id() == stream;
}

struct PackedTensors {
    at::Tensor codes, scales;
    micro_mx4_matrix matrix;
    void make(int64_t rows, int64_t cols, const at::TensorOptions& like) {
        const int64_t groups = (cols + kGroup - 1) / kGroup;
        codes = at::empty({groups, rows, kGroupBytes}, like.dtype(at::kByte));
        scales = at::empty({groups, rows, kGroupBlocks}, like.dtype(at::kByte));
        matrix = {codes.data_ptr(), scales.data_ptr(), rows, cols};
    }
};

// The matrix of a (codes, scales, rows, cols) tuple, whose tensors may have been resized,
// or been given other memory, since they were checked.
bool matrix_of(PyObject* t, int device, micro_mx4_matrix* m) {
    if (!PyTuple_CheckExact(t) || PyTuple_GET_SIZE(t) != 4) return false;
    PyObject *codes = PyTuple_GET_ITEM(t, 0), *scales = PyTuple_GET_ITEM(t, 1);
    if (!THPVariable_CheckExact(codes) || !THPVariable_CheckExact(scales)) return false;
    const at::Tensor &c = THPVariable_Unpack(codes), &s = THPVariable_Unpack(scales);
    const int64_t rows = PyLong_AsLongLong(PyTuple_GET_ITEM(t, 2)), cols = PyLong_AsLongLong(PyTuple_GET_ITEM(t, 3));
    const auto holds = [&](const at::Tensor& x, int64_t bytes) {
        return x.layout() == at::kStrided && x.is_cuda() && x.get_device() == device && x.scalar_type() == at::kByte &&
               x.is_contiguous() && x.dim() == 3 && x.size(0) == (cols + kGroup - 1) / kGroup && x.size(1) == rows &&
               x.size(2) == bytes;
    };
    if (!holds(c, kGroupBytes) || !holds(s, kGroupBlocks)) return false;
    *m = {c.data_ptr(), s.data_ptr(), rows, cols};
    return true;
}

// pack(x, straight, turned): (codes, scales, rows, cols) or None for each of the two;
// None: not the plain case; an int: the call's status.
PyObject* mx_pack(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    MxCaller* c = reinterpret_cast<MxCaller*>(self);
    HANDLE_TH_ERRORS
    if (n != 3 || !THPVariable_CheckExact(args[0])) Py_RETURN_NONE;
    const at::Tensor& x = THPVariable_Unpack(args[0]);
    if (!plain_values(x, c->device) || !on_stream(c->device, c->stream)) Py_RETURN_NONE;
    const int64_t cols = x.size(-1), rows = x.numel() / cols;
    const bool straight = args[1] == Py_True, turned = args[2] == Py_True;
    PackedTensors p, t;
    if (straight) p.make(rows, cols, x.options());
    if (turned) t.make(cols, rows, x.options());
    const void* at = x.data_ptr();
    const int32_t type = type_of(x.scalar_type());
    micro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = c->pack(c->mx, at, type, cols, rows, cols, straight ? &p.matrix : nullptr, turned ? &t.matrix : nullptr);
    Py_END_ALLOW_THREADS
    if (st != MICRO_OK) return PyLong_FromLong(st);
    const auto wrap = [](bool made, PackedTensors& m) -> PyObject* {
        if (!made) return Py_NewRef(Py_None);
        THPObjectPtr codes(THPVariable_Wrap(std::move(m.codes)));
        THPObjectPtr scales(codes.get() ? THPVariable_Wrap(std::move(m.scales)) : nullptr);
        if (!scales.get()) return nullptr;
        return Py_BuildValue("(OOLL)", codes.get(), scales.get(), static_cast<long long>(m.matrix.rows),
                             static_cast<long long>(m.matrix.cols));
    };
    THPObjectPtr first(wrap(straight, p));
    if (!first.get()) return nullptr;
    THPObjectPtr second(wrap(turned, t));
    if (!second.get()) return nullptr;
    return PyTuple_Pack(2, first.get(), second.get());
    END_HANDLE_TH_ERRORS
}

at::ScalarType scalar_of(long type) {
    return type == MICRO_TYPE_F32 ? at::kFloat : type == MICRO_TYPE_F16 ? at::kHalf : at::kBFloat16;
}

// unpack(m, type): the values of a tuple as above in a tensor of its own, of a
// MICRO_TYPE_*; None and an int as above.
PyObject* mx_unpack(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    MxCaller* c = reinterpret_cast<MxCaller*>(self);
    HANDLE_TH_ERRORS
    micro_mx4_matrix m;
    if (n != 2 || !matrix_of(args[0], c->device, &m) || !on_stream(c->device, c->stream)) Py_RETURN_NONE;
    const long type = PyLong_AsLong(args[1]);
    if (type < 0 || type > MICRO_TYPE_BF16) Py_RETURN_NONE;
    at::Tensor out = at::empty({m.rows, m.cols}, THPVariable_Unpack(PyTuple_GET_ITEM(args[0], 0)).options().dtype(scalar_of(type)));
    void* to = out.data_ptr();
    micro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = c->unpack(c->mx, &m, to, static_cast<int32_t>(type), m.cols);
    Py_END_ALLOW_THREADS
    if (st != MICRO_OK) return PyLong_FromLong(st);
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// product(a, b, type): a b^T of two tuples as above into a tensor of its own, of a
// MICRO_TYPE_*; None and an int as above.
PyObject* mx_product(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    MxCaller* c = reinterpret_cast<MxCaller*>(self);
    HANDLE_TH_ERRORS
    micro_mx4_matrix a, b;
    if (n != 3 || !matrix_of(args[0], c->device, &a) || !matrix_of(args[1], c->device, &b) || !on_stream(c->device, c->stream))
        Py_RETURN_NONE;
    const long type = PyLong_AsLong(args[2]);
    if (a.cols != b.cols || type < 0 || type > MICRO_TYPE_BF16) Py_RETURN_NONE;
    at::Tensor out = at::empty({a.rows, b.rows}, THPVariable_Unpack(PyTuple_GET_ITEM(args[0], 0)).options().dtype(scalar_of(type)));
    void* to = out.data_ptr();
    micro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = c->product(c->mx, &a, &b, 0, to, static_cast<int32_t>(type), b.rows);
    Py_END_ALLOW_THREADS
    if (st != MICRO_OK) return PyLong_FromLong(st);
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// linear(x, b, type): x b^T, x packed on the way.
PyObject* mx_linear(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    MxCaller* c = reinterpret_cast<MxCaller*>(self);
    HANDLE_TH_ERRORS
    micro_mx4_matrix b;
    if (n != 3 || !THPVariable_CheckExact(args[0]) || !matrix_of(args[1], c->device, &b)) Py_RETURN_NONE;
    const at::Tensor& x = THPVariable_Unpack(args[0]);
    if (!plain_values(x, c->device) || x.size(-1) != b.cols || !on_stream(c->device, c->stream)) Py_RETURN_NONE;
    const long type = PyLong_AsLong(args[2]);
    if (type < 0 || type > MICRO_TYPE_BF16) Py_RETURN_NONE;
    PackedTensors p;
    p.make(x.numel() / b.cols, b.cols, x.options());
    c10::SmallVector<int64_t, 6> shape(x.sizes().begin(), x.sizes().end());
    shape.back() = b.rows;
    at::Tensor out = at::empty(shape, x.options().dtype(scalar_of(type)));
    const void* from = x.data_ptr();
    void* to = out.data_ptr();
    const int32_t x_type = type_of(x.scalar_type());
    micro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = c->linear(c->mx, from, x_type, b.cols, &p.matrix, &b, 0, to, static_cast<int32_t>(type), b.rows);
    Py_END_ALLOW_THREADS
    if (st != MICRO_OK) return PyLong_FromLong(st);
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// MxCaller(pack, unpack, product, linear, mx, device, stream).
PyObject* mx_caller_new(PyTypeObject* type, PyObject* args, PyObject*) {
    unsigned long long pack, unpack, product, linear, mx;
    int device;
    long long stream;
    if (!PyArg_ParseTuple(args, "KKKKKiL", &pack, &unpack, &product, &linear, &mx, &device, &stream)) return nullptr;
    MxCaller* c = reinterpret_cast<MxCaller*>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    c->pack = reinterpret_cast<decltype(c->pack)>(pack);
    c->unpack = reinterpret_cast<decltype(c->unpack)>(unpack);
    c->product = reinterpret_cast<decltype(c->product)>(product);
    c->linear = reinterpret_cast<decltype(c->linear)>(linear);
    c->mx = reinterpret_cast<micro_mx4*>(mx);
    c->device = device;
    c->stream = stream;
    return reinterpret_cast<PyObject*>(c);
}

PyMethodDef mx_methods[] = {
    {"pack", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(mx_pack)), METH_FASTCALL, nullptr},
    {"unpack", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(mx_unpack)), METH_FASTCALL, nullptr},
    {"product", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(mx_product)), METH_FASTCALL, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(mx_linear)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject mx_caller_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyMethodDef caller_methods[] = {
    {"step", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(caller_step)), METH_FASTCALL, nullptr},
    {"ef_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(caller_ef_step)), METH_FASTCALL, nullptr},
    {"sweep", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(caller_sweep)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject caller_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_caller", nullptr, -1, nullptr, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__caller() {
    caller_type.tp_name = "paper_2310_00967_amd._caller.Caller";
    caller_type.tp_basicsize = sizeof(Caller);
    caller_type.tp_flags = Py_TPFLAGS_DEFAULT;
    caller_type.tp_methods = caller_methods;
    caller_type.tp_new = caller_new;
    if (PyType_Ready(&caller_type) < 0) return nullptr;
    table_caller_type.tp_name = "paper_2310_00967_amd._caller.TableCaller";
    table_caller_type.tp_basicsize = sizeof(TableCaller);
    table_caller_type.tp_flags = Py_TPFLAGS_DEFAULT;
    table_caller_type.tp_methods = table_methods;
    table_caller_type.tp_new = table_caller_new;
    if (PyType_Ready(&table_caller_type) < 0) return nullptr;
    mx_caller_type.tp_name = "paper_2310_00967_amd._caller.MxCaller";
    mx_caller_type.tp_basicsize = sizeof(MxCaller);
    mx_caller_type.tp_flags = Py_TPFLAGS_DEFAULT;
    mx_caller_type.tp_methods = mx_methods;
    mx_caller_type.tp_new = mx_caller_new;
    if (PyType_Ready(&mx_caller_type) < 0) return nullptr;
    PyObject* m = PyModule_Create(&module);
    if (!m) return nullptr;
    if (PyModule_AddObject(m, "Caller", Py_NewRef(reinterpret_cast<PyObject*>(&caller_type))) < 0 ||
        PyModule_AddObject(m, "TableCaller", Py_NewRef(reinterpret_cast<PyObject*>(&table_caller_type))) < 0 ||
        PyModule_AddObject(m, "MxCaller", Py_NewRef(reinterpret_cast<PyObject*>(&mx_caller_type))) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}

// Python entry of the calls that a program makes every step: selection,
// collection, priority update and their sharded forms, and the learner's
// operators on collected windows, whose tensors it checks.
//
// A step's kernels take 2 to 20 us on the small workloads, and allocating its
// outputs and marshalling its arguments in Python took longer than that.  Each
// function here allocates the outputs as torch tensors, passes their addresses
// to the C ABI and wraps them, with the interpreter lock released around the
// library call.  The library is reached through the addresses that the Python
// binding hands to bind(), so both use the one it loaded.
//
// Every call returns its results, or the library's negative status as an int.
#include <Python.h>

#include <ATen/Functions.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>
#include <vector>

#include "gear.h"

namespace {

decltype(&gear_select) f_select = nullptr;
decltype(&gear_collect) f_collect = nullptr;
decltype(&gear_select_collect) f_select_collect = nullptr;
decltype(&gear_update_priorities) f_update = nullptr;
decltype(&gear_select_shard) f_select_shard = nullptr;
decltype(&gear_is_weights) f_is_weights = nullptr;
decltype(&gear_topk_merge) f_topk_merge = nullptr;
decltype(&gear_recurrence_sizes) f_recurrence_sizes = nullptr;
decltype(&gear_recurrence) f_recurrence = nullptr;
decltype(&gear_recurrence_backward) f_recurrence_backward = nullptr;
decltype(&gear_advantages_sizes) f_advantages_sizes = nullptr;
decltype(&gear_advantages) f_advantages = nullptr;
decltype(&gear_policy_sizes) f_policy_sizes = nullptr;
decltype(&gear_policy_loss) f_policy_loss = nullptr;
decltype(&gear_action_logp) f_action_logp = nullptr;

// One column of a table as its batches are handed out.
struct Column {
    at::ScalarType dtype;
    std::vector<int64_t> shape;  // per step
    int64_t elem_bytes;
};
const char* const kPlanName = "gear column plan";

// A Python error that is already set.
struct PythonError {};

int64_t as_int(PyObject* o) {
    PyObject* i = PyNumber_Index(o);
    if (i == nullptr) throw PythonError();
    const long long v = PyLong_AsLongLong(i);
    Py_DECREF(i);
    if (v == -1 && PyErr_Occurred()) throw PythonError();
    return v;
}

int32_t as_int32(PyObject* o) {
    const int64_t v = as_int(o);
    if (v != (int32_t)v) {
        PyErr_SetString(PyExc_OverflowError, "argument out of the 32-bit range");
        throw PythonError();
    }
    return (int32_t)v;
}

uint64_t as_u64(PyObject* o) {
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw PythonError();
    return v;
}

float as_float(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError();
    return (float)v;
}

bool as_bool(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError();
    return v != 0;
}

void* as_ptr(PyObject* o) {
    if (o == Py_None) return nullptr;
    void* p = PyLong_AsVoidPtr(o);
    if (p == nullptr && PyErr_Occurred()) throw PythonError();
    return p;
}

// Device address of a tensor, or of anything else with a data_ptr() method.
void* address_of(PyObject* o) {
    if (THPVariable_Check(o)) return THPVariable_Unpack(o).data_ptr();
    PyObject* v = PyObject_CallMethod(o, "data_ptr", nullptr);
    if (v == nullptr) throw PythonError();
    void* p = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    if (p == nullptr && PyErr_Occurred()) throw PythonError();
    return p;
}

// shape[0], which the library takes as a 32-bit batch size.
int32_t batch_of(PyObject* o) {
    int64_t n;
    if (THPVariable_Check(o)) {
        n = THPVariable_Unpack(o).size(0);
    } else {
        PyObject* shape = PyObject_GetAttrString(o, "shape");
        if (shape == nullptr) throw PythonError();
        PyObject* v = PySequence_GetItem(shape, 0);
        Py_DECREF(shape);
        if (v == nullptr) throw PythonError();
        n = PyLong_AsLongLong(v);
        Py_DECREF(v);
        if (n == -1 && PyErr_Occurred()) throw PythonError();
    }
    if (n != (int32_t)n) {
        PyErr_SetString(PyExc_OverflowError, "batch out of the 32-bit range");
        throw PythonError();
    }
    return (int32_t)n;
}

at::Tensor empty(at::IntArrayRef sizes, at::ScalarType dtype, int32_t device) {
    return at::empty(sizes, at::TensorOptions().dtype(dtype).device(at::Device(at::kCUDA, (at::DeviceIndex)device)));
}

PyObject* wrap(at::Tensor t) {
    PyObject* o = THPVariable_Wrap(std::move(t));
    if (o == nullptr) throw PythonError();
    return o;
}

template <typename F>
int without_gil(F call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}

// A tuple that owns the items set so far.
struct Tuple {
    PyObject* t;
    explicit Tuple(Py_ssize_t n) : t(PyTuple_New(n)) {
        if (t == nullptr) throw PythonError();
    }
    ~Tuple() { Py_XDECREF(t); }
    void set(Py_ssize_t i, PyObject* o) { PyTuple_SET_ITEM(t, i, o); }
    void none(Py_ssize_t i) {
        Py_INCREF(Py_None);
        PyTuple_SET_ITEM(t, i, Py_None);
    }
    PyObject* release() {
        PyObject* r = t;
        t = nullptr;
        return r;
    }
};

// The batch buffers of a call: `ids` None for every column, else a list.
struct Batch {
    std::vector<int32_t> ids;
    std::vector<at::Tensor> out;
    std::vector<void*> ptr;
    bool all;

    Batch(PyObject* plan, PyObject* id_list, bool typed, int64_t B, int64_t L, int32_t device) {
        const auto* cols = static_cast<const std::vector<Column>*>(PyCapsule_GetPointer(plan, kPlanName));
        if (cols == nullptr) throw PythonError();
        all = id_list == Py_None;
        if (all) {
            for (size_t c = 0; c < cols->size(); c++) ids.push_back((int32_t)c);
        } else {
            const Py_ssize_t n = PyList_Size(id_list);
            if (n < 0) throw PythonError();
            for (Py_ssize_t k = 0; k < n; k++) {
                int64_t c = as_int(PyList_GET_ITEM(id_list, k));
                // Sizes come from Python's indexing (from the end when
                // negative); the library checks the number itself.
                const int64_t have = (int64_t)cols->size();
                if (c < -have || c >= have) {
                    PyErr_SetString(PyExc_IndexError, "list index out of range");
                    throw PythonError();
                }
                ids.push_back((int32_t)c);
            }
        }
        std::vector<int64_t> sizes;
        for (int32_t id : ids) {
            const Column& c = (*cols)[id < 0 ? id + (int32_t)cols->size() : id];
            if (typed) {
                sizes.assign({B, L});
                sizes.insert(sizes.end(), c.shape.begin(), c.shape.end());
                out.push_back(empty(sizes, c.dtype, device));
            } else {
                out.push_back(empty({B, L * c.elem_bytes}, at::kByte, device));
            }
            ptr.push_back(out.back().data_ptr());
        }
    }
    const int32_t* id_data() const { return all ? nullptr : ids.data(); }
    PyObject* list() {
        PyObject* l = PyList_New((Py_ssize_t)out.size());
        if (l == nullptr) throw PythonError();
        for (size_t k = 0; k < out.size(); k++) {
            PyObject* o = THPVariable_Wrap(out[k]);
            if (o == nullptr) {
                Py_DECREF(l);
                throw PythonError();
            }
            PyList_SET_ITEM(l, (Py_ssize_t)k, o);
        }
        return l;
    }
};

// Every entry: argument count, and C++ exceptions turned into Python ones.
template <typename F>
PyObject* entry(Py_ssize_t have, Py_ssize_t want, F body) {
    if (have != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, have);
        return nullptr;
    }
    HANDLE_TH_ERRORS
    try {
        return body();
    } catch (const PythonError&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 15, [&]() -> PyObject* {
        f_select = reinterpret_cast<decltype(f_select)>(as_ptr(a[0]));
        f_collect = reinterpret_cast<decltype(f_collect)>(as_ptr(a[1]));
        f_select_collect = reinterpret_cast<decltype(f_select_collect)>(as_ptr(a[2]));
        f_update = reinterpret_cast<decltype(f_update)>(as_ptr(a[3]));
        f_select_shard = reinterpret_cast<decltype(f_select_shard)>(as_ptr(a[4]));
        f_is_weights = reinterpret_cast<decltype(f_is_weights)>(as_ptr(a[5]));
        f_topk_merge = reinterpret_cast<decltype(f_topk_merge)>(as_ptr(a[6]));
        f_recurrence_sizes = reinterpret_cast<decltype(f_recurrence_sizes)>(as_ptr(a[7]));
        f_recurrence = reinterpret_cast<decltype(f_recurrence)>(as_ptr(a[8]));
        f_recurrence_backward = reinterpret_cast<decltype(f_recurrence_backward)>(as_ptr(a[9]));
        f_advantages_sizes = reinterpret_cast<decltype(f_advantages_sizes)>(as_ptr(a[10]));
        f_advantages = reinterpret_cast<decltype(f_advantages)>(as_ptr(a[11]));
        f_policy_sizes = reinterpret_cast<decltype(f_policy_sizes)>(as_ptr(a[12]));
        f_policy_loss = reinterpret_cast<decltype(f_policy_loss)>(as_ptr(a[13]));
        f_action_logp = reinterpret_cast<decltype(f_action_logp)>(as_ptr(a[14]));
        Py_RETURN_NONE;
    });
}

// plan([(dtype, shape, elem_bytes), ...])
PyObject* py_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 1, [&]() -> PyObject* {
        auto cols = std::make_unique<std::vector<Column>>();
        const Py_ssize_t k = PyList_Size(a[0]);
        if (k < 0) throw PythonError();
        for (Py_ssize_t i = 0; i < k; i++) {
            PyObject *dtype, *shape;
            long long eb;
            if (!PyArg_ParseTuple(PyList_GET_ITEM(a[0], i), "O!O!L", &THPDtypeType, &dtype, &PyTuple_Type, &shape, &eb))
                throw PythonError();
            Column c;
            c.dtype = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
            for (Py_ssize_t d = 0; d < PyTuple_GET_SIZE(shape); d++) c.shape.push_back(as_int(PyTuple_GET_ITEM(shape, d)));
            c.elem_bytes = eb;
            cols->push_back(std::move(c));
        }
        PyObject* cap = PyCapsule_New(cols.get(), kPlanName, [](PyObject* o) {
            delete static_cast<std::vector<Column>*>(PyCapsule_GetPointer(o, kPlanName));
        });
        if (cap == nullptr) throw PythonError();
        cols.release();
        return cap;
    });
}

// select(handle, strategy, B, L, seed, beta, weights, device, stream)
PyObject* py_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 9, [&]() -> PyObject* {
        gear_table* t = static_cast<gear_table*>(as_ptr(a[0]));
        const int32_t strategy = as_int32(a[1]), B = as_int32(a[2]), L = as_int32(a[3]), dev = as_int32(a[7]);
        const uint64_t seed = as_u64(a[4]);
        const float beta = as_float(a[5]);
        const bool weights = as_bool(a[6]);
        void* s = as_ptr(a[8]);
        at::Tensor idx = empty({B}, at::kLong, dev), start = empty({B}, at::kInt, dev), w;
        if (weights) w = empty({B}, at::kFloat, dev);
        int64_t* pi = static_cast<int64_t*>(idx.data_ptr());
        int32_t* ps = static_cast<int32_t*>(start.data_ptr());
        float* pw = weights ? static_cast<float*>(w.data_ptr()) : nullptr;
        const int rc = without_gil([&] { return f_select(t, strategy, B, L, seed, beta, pi, ps, pw, s); });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        Tuple r(3);
        r.set(0, wrap(std::move(idx)));
        r.set(1, wrap(std::move(start)));
        if (weights) r.set(2, wrap(std::move(w)));
        else r.none(2);
        return r.release();
    });
}

// collect(handle, plan, idx, start, L, ids, typed, device, stream): list of batches
PyObject* py_collect(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 9, [&]() -> PyObject* {
        gear_table* t = static_cast<gear_table*>(as_ptr(a[0]));
        const int32_t B = batch_of(a[2]), L = as_int32(a[4]), dev = as_int32(a[7]);
        void* s = as_ptr(a[8]);
        Batch batch(a[1], a[5], as_bool(a[6]), B, L, dev);
        const int64_t* pi = static_cast<const int64_t*>(address_of(a[2]));
        const int32_t* ps = static_cast<const int32_t*>(address_of(a[3]));
        const int rc = without_gil([&] {
            return f_collect(t, pi, ps, B, L, batch.id_data(), (int32_t)batch.ptr.size(), batch.ptr.data(), s);
        });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        return batch.list();
    });
}

// select_collect(handle, plan, strategy, B, L, seed, weights, ids, typed, device, stream)
PyObject* py_select_collect(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 11, [&]() -> PyObject* {
        gear_table* t = static_cast<gear_table*>(as_ptr(a[0]));
        const int32_t strategy = as_int32(a[2]), B = as_int32(a[3]), L = as_int32(a[4]), dev = as_int32(a[9]);
        const uint64_t seed = as_u64(a[5]);
        const bool weights = as_bool(a[6]);
        void* s = as_ptr(a[10]);
        at::Tensor idx = empty({B}, at::kLong, dev), start = empty({B}, at::kInt, dev), w;
        if (weights) w = empty({B}, at::kFloat, dev);
        Batch batch(a[1], a[7], as_bool(a[8]), B, L, dev);
        int64_t* pi = static_cast<int64_t*>(idx.data_ptr());
        int32_t* ps = static_cast<int32_t*>(start.data_ptr());
        float* pw = weights ? static_cast<float*>(w.data_ptr()) : nullptr;
        const int rc = without_gil([&] {
            return f_select_collect(t, strategy, B, L, seed, pi, ps, pw, batch.id_data(), (int32_t)batch.ptr.size(),
                                    batch.ptr.data(), s);
        });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        Tuple r(4);
        r.set(0, wrap(std::move(idx)));
        r.set(1, wrap(std::move(start)));
        if (weights) r.set(2, wrap(std::move(w)));
        else r.none(2);
        r.set(3, batch.list());
        return r.release();
    });
}

// update(handle, idx, new, stream)
PyObject* py_update(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 4, [&]() -> PyObject* {
        gear_table* t = static_cast<gear_table*>(as_ptr(a[0]));
        void* s = as_ptr(a[3]);
        const int32_t B = batch_of(a[1]);
        const int64_t* pi = static_cast<const int64_t*>(address_of(a[1]));
        const uint32_t* pp = static_cast<const uint32_t*>(address_of(a[2]));
        return PyLong_FromLong(without_gil([&] { return f_update(t, pi, pp, B, s); }));
    });
}

// select_shard(handle, G, g, totals, base, B, L, seed, device, stream)
PyObject* py_select_shard(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 10, [&]() -> PyObject* {
        gear_table* t = static_cast<gear_table*>(as_ptr(a[0]));
        const int32_t G = as_int32(a[1]), g = as_int32(a[2]), B = as_int32(a[5]), L = as_int32(a[6]);
        const int64_t base = as_int(a[4]);
        const uint64_t seed = as_u64(a[7]);
        const int32_t dev = as_int32(a[8]);
        void* s = as_ptr(a[9]);
        const uint64_t* totals = static_cast<const uint64_t*>(address_of(a[3]));
        at::Tensor idx = empty({B}, at::kLong, dev), start = empty({B}, at::kInt, dev), p = empty({B}, at::kInt, dev);
        int64_t* pi = static_cast<int64_t*>(idx.data_ptr());
        int32_t* ps = static_cast<int32_t*>(start.data_ptr());
        uint32_t* pp = static_cast<uint32_t*>(p.data_ptr());
        const int rc = without_gil([&] { return f_select_shard(t, G, g, totals, base, B, L, seed, pi, ps, pp, s); });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        Tuple r(3);
        r.set(0, wrap(std::move(idx)));
        r.set(1, wrap(std::move(start)));
        r.set(2, wrap(std::move(p)));
        return r.release();
    });
}

// is_weights(handle, sel_prio, beta, device, stream)
PyObject* py_is_weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 5, [&]() -> PyObject* {
        gear_table* t = static_cast<gear_table*>(as_ptr(a[0]));
        const float beta = as_float(a[2]);
        const int32_t B = batch_of(a[1]), dev = as_int32(a[3]);
        void* s = as_ptr(a[4]);
        at::Tensor w = empty({B}, at::kFloat, dev);
        const uint32_t* pp = static_cast<const uint32_t*>(address_of(a[1]));
        float* pw = static_cast<float*>(w.data_ptr());
        const int rc = without_gil([&] { return f_is_weights(t, pp, B, beta, pw, s); });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        return wrap(std::move(w));
    });
}

// topk_merge(prio, gidx, G, K, T, L, seed, device, stream)
PyObject* py_topk_merge(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 9, [&]() -> PyObject* {
        const uint32_t* p = static_cast<const uint32_t*>(address_of(a[0]));
        const int64_t* gi = static_cast<const int64_t*>(address_of(a[1]));
        const int32_t G = as_int32(a[2]), K = as_int32(a[3]), T = as_int32(a[4]), L = as_int32(a[5]);
        const uint64_t seed = as_u64(a[6]);
        const int32_t dev = as_int32(a[7]);
        void* s = as_ptr(a[8]);
        at::Tensor idx = empty({K}, at::kLong, dev), start = empty({K}, at::kInt, dev);
        at::Tensor w = empty({K}, at::kFloat, dev), q = empty({K}, at::kInt, dev);
        int64_t* pi = static_cast<int64_t*>(idx.data_ptr());
        int32_t* ps = static_cast<int32_t*>(start.data_ptr());
        float* pw = static_cast<float*>(w.data_ptr());
        uint32_t* pq = static_cast<uint32_t*>(q.data_ptr());
        const int rc = without_gil([&] { return f_topk_merge(p, gi, G, K, T, L, seed, pi, ps, pw, pq, s); });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        Tuple r(4);
        r.set(0, wrap(std::move(idx)));
        r.set(1, wrap(std::move(start)));
        r.set(2, wrap(std::move(w)));
        r.set(3, wrap(std::move(q)));
        return r.release();
    });
}

// ---------------------------------------------------------------------------
// The learner's operators.  Their tensors come from a model, so unlike the
// calls above these check types, shapes, strides and devices (ValueError).
// ---------------------------------------------------------------------------

using Sizes = std::vector<int64_t>;

const at::Tensor& tensor_of(PyObject* o, const char* name) {
    TORCH_CHECK_TYPE(THPVariable_Check(o), name, " must be a torch tensor");
    return THPVariable_Unpack(o);
}

void need_device(const at::Tensor& t, const char* name, c10::Device dev) {
    TORCH_CHECK_VALUE(t.device() == dev, name, " must be on ", dev, ", not ", t.device());
}

// GEAR_DTYPE_* of a floating-point tensor.
int32_t float_code(const at::Tensor& t, const char* name) {
    switch (t.scalar_type()) {
        case at::kFloat: return GEAR_DTYPE_F32;
        case at::kBFloat16: return GEAR_DTYPE_BF16;
        case at::kHalf: return GEAR_DTYPE_F16;
        default: TORCH_CHECK_VALUE(false, name, " must be float32, bfloat16 or float16, not ", t.scalar_type());
    }
}

void need_sizes(const at::Tensor& t, const char* name, const Sizes& want) {
    TORCH_CHECK_VALUE(t.sizes() == at::IntArrayRef(want), name, " must have shape ", at::IntArrayRef(want), ", not ",
                      t.sizes());
}

// Elements of the last dimension lie next to each other.
void need_rows(const at::Tensor& t, const char* name) {
    TORCH_CHECK_VALUE(t.dim() > 0 && (t.size(-1) <= 1 || t.stride(-1) == 1), name,
                      " must be contiguous along its last dimension");
}

// A tensor or None: contiguous, of one of the byte flag types (uint8, bool) or of `dtype`.
enum class Kind { kFlags, kInt32, kFloat };
at::Tensor optional_of(PyObject* o, const char* name, Kind kind, c10::Device dev) {
    if (o == Py_None) return at::Tensor();
    const at::Tensor& t = tensor_of(o, name);
    need_device(t, name, dev);
    if (kind == Kind::kFlags) {
        TORCH_CHECK_VALUE(t.scalar_type() == at::kByte || t.scalar_type() == at::kBool, name,
                          " must be uint8 or bool, not ", t.scalar_type());
    } else if (kind == Kind::kInt32) {
        TORCH_CHECK_VALUE(t.scalar_type() == at::kInt, name, " must be int32, not ", t.scalar_type());
    } else {
        TORCH_CHECK_VALUE(t.scalar_type() == at::kFloat, name, " must be float32, not ", t.scalar_type());
    }
    return t;
}
void need_contiguous(const at::Tensor& t, const char* name) {
    TORCH_CHECK_VALUE(!t.defined() || t.is_contiguous(), name, " must be contiguous");
}

template <typename T>
T* data(const at::Tensor& t) {
    return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr;
}

at::Tensor make(at::IntArrayRef sizes, at::ScalarType dtype, c10::Device dev) {
    return at::empty(sizes, at::TensorOptions().dtype(dtype).device(dev));
}

// Workspace of so many bytes; undefined for none.  It returns to torch's
// allocator when the call has been enqueued, for work on the same stream.
at::Tensor workspace(int64_t bytes, c10::Device dev) {
    return bytes > 0 ? make({bytes}, at::kByte, dev) : at::Tensor();
}

// Tells autograd that a call writes over a tensor of the caller's: a gradient that
// needs what it held is then refused.  Inference tensors have no versions, and no gradient needs them.
void overwrites(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// Refuses an input that lies in the memory of `out`, which is contiguous and
// which the call writes: other lanes may read the input afterwards.  The input is
// contiguous, or has one or two dimensions and contiguous rows.
void need_apart(const at::Tensor& out, const char* out_name, const at::Tensor& t, const char* name) {
    if (!t.defined() || t.numel() == 0 || out.numel() == 0) return;
    const char *o = data<char>(out), *o_end = o + out.nbytes(), *p = data<char>(t);
    const int64_t item = t.element_size();
    int64_t rows = 1, stride = 0, run = t.numel() * item;
    if (!t.is_contiguous()) {
        rows = t.size(0);
        stride = t.stride(0) * item;
        run = t.dim() == 2 ? t.size(1) * item : item;
    }
    bool meet = o < p + (rows - 1) * stride + run && p < o_end;
    if (meet && rows > 1) {
        meet = false;
        for (int64_t r = 0; r < rows; r++) meet |= o < p + r * stride + run && p + r * stride < o_end;
    }
    TORCH_CHECK_VALUE(!meet, name, " must not overlap ", out_name, ", which is written");
}

c10::Device gpu_of(const at::Tensor& t, const char* name) {
    TORCH_CHECK_VALUE(t.is_cuda(), name, " must be on the GPU, not on ", t.device());
    return t.device();
}

// What both directions of the recurrence take.
struct Recurrence {
    at::Tensor gate, x, state, reset, lengths;
    gear_recurrence_desc d{};
    c10::Device dev = c10::Device(at::kCPU);

    Recurrence(PyObject* o_gate, PyObject* o_x, PyObject* o_state, PyObject* o_form, PyObject* o_reset,
               PyObject* o_lengths, bool step) {
        gate = tensor_of(o_gate, "gate");
        x = tensor_of(o_x, "x");
        dev = gpu_of(x, "x");
        need_device(gate, "gate", dev);
        d.dtype = float_code(x, "x");
        TORCH_CHECK_VALUE(gate.scalar_type() == x.scalar_type(), "gate and x must have one dtype");
        if (step) {
            TORCH_CHECK_VALUE(x.dim() == 2, "x must have shape [B, D], not ", x.sizes());
        } else {
            TORCH_CHECK_VALUE(x.dim() == 3, "x must have shape [B, T, D], not ", x.sizes());
        }
        need_sizes(gate, "gate", x.sizes().vec());
        need_rows(gate, "gate");
        need_rows(x, "x");
        d.form = as_int32(o_form);
        d.B = x.size(0);
        d.T = step ? 1 : x.size(1);
        d.D = x.size(-1);
        d.gate_b = gate.stride(0);
        d.gate_t = step ? 0 : gate.stride(1);
        d.x_b = x.stride(0);
        d.x_t = step ? 0 : x.stride(1);
        state = optional_of(o_state, "state", Kind::kFloat, dev);
        if (state.defined()) need_sizes(state, "state", {d.B, d.D});
        need_contiguous(state, "state");
        reset = optional_of(o_reset, "reset", Kind::kFlags, dev);
        if (reset.defined()) {
            need_sizes(reset, "reset", step ? Sizes{d.B} : Sizes{d.B, d.T});
            if (!step) need_rows(reset, "reset");
            d.reset_b = reset.stride(0);
        }
        lengths = optional_of(o_lengths, "lengths", Kind::kInt32, dev);
        if (lengths.defined()) need_sizes(lengths, "lengths", {d.B});
        need_contiguous(lengths, "lengths");
        d.d_reset = data<uint8_t>(reset);
        d.d_lengths = data<int32_t>(lengths);
    }
};

// recurrence(gate, x, state, form, reset, lengths, save, stream): (y, final, saved or None)
PyObject* py_recurrence(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 8, [&]() -> PyObject* {
        const Recurrence r(a[0], a[1], a[2], a[3], a[4], a[5], false);
        const bool save = as_bool(a[6]);
        void* s = as_ptr(a[7]);
        const c10::DeviceGuard guard(r.dev);
        int64_t saved_bytes = 0, work_bytes = 0;
        int rc = f_recurrence_sizes(&r.d, &saved_bytes, &work_bytes);
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        at::Tensor y = make({r.d.B, r.d.T, r.d.D}, r.x.scalar_type(), r.dev);
        at::Tensor last = make({r.d.B, r.d.D}, at::kFloat, r.dev), saved;
        if (save) saved = make({saved_bytes / 4}, at::kFloat, r.dev);
        const at::Tensor work = workspace(work_bytes, r.dev);
        rc = without_gil([&] {
            return f_recurrence(&r.d, r.gate.data_ptr(), r.x.data_ptr(), data<float>(r.state), y.data_ptr(),
                                data<float>(last), data<float>(saved), data<void>(work), work_bytes, s);
        });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        Tuple t(3);
        t.set(0, wrap(std::move(y)));
        t.set(1, wrap(std::move(last)));
        if (save) t.set(2, wrap(std::move(saved)));
        else t.none(2);
        return t.release();
    });
}

// recurrence_step(gate, x, state, form, reset, out, stream): (y, state)
PyObject* py_recurrence_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 7, [&]() -> PyObject* {
        const Recurrence r(a[0], a[1], a[2], a[3], a[4], Py_None, true);
        void* s = as_ptr(a[6]);
        const c10::DeviceGuard guard(r.dev);
        at::Tensor out = optional_of(a[5], "out", Kind::kFloat, r.dev);
        if (out.defined()) need_sizes(out, "out", {r.d.B, r.d.D});
        else out = make({r.d.B, r.d.D}, at::kFloat, r.dev);
        need_contiguous(out, "out");
        if (r.state.defined() && out.data_ptr() != r.state.data_ptr()) {
            const char *p = data<char>(out), *q = data<char>(r.state);
            const int64_t bytes = r.d.B * r.d.D * 4;
            TORCH_CHECK_VALUE(p + bytes <= q || q + bytes <= p, "out must be state itself or not overlap it");
        }
        if (a[5] != Py_None) {
            need_apart(out, "out", r.gate, "gate");
            need_apart(out, "out", r.x, "x");
            need_apart(out, "out", r.reset, "reset");
        }
        at::Tensor y = make({r.d.B, r.d.D}, r.x.scalar_type(), r.dev);
        if (a[5] != Py_None) overwrites(out);
        const int rc = without_gil([&] {
            return f_recurrence(&r.d, r.gate.data_ptr(), r.x.data_ptr(), data<float>(r.state), y.data_ptr(),
                                data<float>(out), nullptr, nullptr, 0, s);
        });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        Tuple t(2);
        t.set(0, wrap(std::move(y)));
        t.set(1, wrap(std::move(out)));
        return t.release();
    });
}

// recurrence_backward(gate, x, state, form, reset, lengths, saved, dy, dfinal, stream): (dgate, dx, dstate)
PyObject* py_recurrence_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 10, [&]() -> PyObject* {
        Recurrence r(a[0], a[1], a[2], a[3], a[4], a[5], false);
        void* s = as_ptr(a[9]);
        const c10::DeviceGuard guard(r.dev);
        int64_t saved_bytes = 0, work_bytes = 0;
        int rc = f_recurrence_sizes(&r.d, &saved_bytes, &work_bytes);
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        const at::Tensor saved = optional_of(a[6], "saved", Kind::kFloat, r.dev);
        TORCH_CHECK_VALUE(saved.defined(), "saved must be what recurrence(..., save=True) returned");
        need_sizes(saved, "saved", {saved_bytes / 4});
        need_contiguous(saved, "saved");
        at::Tensor dy;
        if (a[7] != Py_None) {
            dy = tensor_of(a[7], "dy");
            need_device(dy, "dy", r.dev);
            TORCH_CHECK_VALUE(dy.scalar_type() == r.x.scalar_type(), "dy and x must have one dtype");
            need_sizes(dy, "dy", r.x.sizes().vec());
            need_rows(dy, "dy");
            r.d.dy_b = dy.stride(0);
            r.d.dy_t = dy.stride(1);
        }
        const at::Tensor dfinal = optional_of(a[8], "dfinal", Kind::kFloat, r.dev);
        if (dfinal.defined()) need_sizes(dfinal, "dfinal", {r.d.B, r.d.D});
        need_contiguous(dfinal, "dfinal");
        at::Tensor dgate = make(r.x.sizes(), r.x.scalar_type(), r.dev), dx = make(r.x.sizes(), r.x.scalar_type(), r.dev);
        at::Tensor dstate = make({r.d.B, r.d.D}, at::kFloat, r.dev);
        const at::Tensor work = workspace(work_bytes, r.dev);
        rc = without_gil([&] {
            return f_recurrence_backward(&r.d, r.gate.data_ptr(), r.x.data_ptr(), data<float>(r.state), data<float>(saved),
                                         data<void>(dy), data<float>(dfinal), dgate.data_ptr(), dx.data_ptr(),
                                         data<float>(dstate), data<void>(work), work_bytes, s);
        });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        Tuple t(3);
        t.set(0, wrap(std::move(dgate)));
        t.set(1, wrap(std::move(dx)));
        t.set(2, wrap(std::move(dstate)));
        return t.release();
    });
}

// advantages(reward, value, gamma, lambda, done, lengths, stream): (adv, ret)
PyObject* py_advantages(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 7, [&]() -> PyObject* {
        const at::Tensor& reward = tensor_of(a[0], "reward");
        const at::Tensor& value = tensor_of(a[1], "value");
        const c10::Device dev = gpu_of(reward, "reward");
        need_device(value, "value", dev);
        gear_advantages_desc d{};
        d.reward_dtype = float_code(reward, "reward");
        d.value_dtype = float_code(value, "value");
        TORCH_CHECK_VALUE(reward.dim() == 2, "reward must have shape [B, L], not ", reward.sizes());
        d.B = reward.size(0);
        d.L = reward.size(1);
        need_sizes(value, "value", {d.B, d.L + 1});
        need_rows(reward, "reward");
        need_rows(value, "value");
        d.reward_b = reward.stride(0);
        d.value_b = value.stride(0);
        d.gamma = as_float(a[2]);
        d.lambda = as_float(a[3]);
        const at::Tensor done = optional_of(a[4], "done", Kind::kFlags, dev);
        if (done.defined()) {
            need_sizes(done, "done", {d.B, d.L});
            need_rows(done, "done");
            d.done_b = done.stride(0);
        }
        const at::Tensor lengths = optional_of(a[5], "lengths", Kind::kInt32, dev);
        if (lengths.defined()) need_sizes(lengths, "lengths", {d.B});
        need_contiguous(lengths, "lengths");
        d.d_done = data<uint8_t>(done);
        d.d_lengths = data<int32_t>(lengths);
        void* s = as_ptr(a[6]);
        const c10::DeviceGuard guard(dev);
        int64_t work_bytes = 0;
        int rc = f_advantages_sizes(&d, &work_bytes);
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        at::Tensor adv = make({d.B, d.L}, at::kFloat, dev), ret = make({d.B, d.L}, at::kFloat, dev);
        const at::Tensor work = workspace(work_bytes, dev);
        rc = without_gil([&] {
            return f_advantages(&d, reward.data_ptr(), value.data_ptr(), data<float>(adv), data<float>(ret),
                                data<void>(work), work_bytes, s);
        });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        Tuple t(2);
        t.set(0, wrap(std::move(adv)));
        t.set(1, wrap(std::move(ret)));
        return t.release();
    });
}

// Logits [..., V], the actions taken and a mask of them.
struct Policy {
    at::Tensor logits, action, mask;
    gear_policy_desc d{};
    c10::Device dev = c10::Device(at::kCPU);
    Sizes rows;  // the logits' leading sizes

    // Consecutive rows that share a value of `t`, whose shape is the first of the leading sizes.
    int64_t group_of(const at::Tensor& t, const char* name) const {
        TORCH_CHECK_VALUE(t.dim() >= 1 || rows.empty(), name, " must have at least one dimension");
        TORCH_CHECK_VALUE((size_t)t.dim() <= rows.size(), name, " has more dimensions than action");
        int64_t g = 1;
        for (size_t i = 0; i < rows.size(); i++) {
            if (i < (size_t)t.dim()) {
                TORCH_CHECK_VALUE(t.size((int64_t)i) == rows[i], name, " must have the first sizes of ",
                                  at::IntArrayRef(rows), ", not ", t.sizes());
            } else {
                g *= rows[i];
            }
        }
        return g < 1 ? 1 : g;
    }

    Policy(PyObject* o_logits, PyObject* o_action, PyObject* o_mask) {
        logits = tensor_of(o_logits, "logits");
        action = tensor_of(o_action, "action");
        dev = gpu_of(logits, "logits");
        need_device(action, "action", dev);
        d.dtype = float_code(logits, "logits");
        TORCH_CHECK_VALUE(logits.dim() >= 2, "logits must have shape [..., V] with at least one row dimension");
        need_rows(logits, "logits");
        d.V = logits.size(-1);
        TORCH_CHECK_VALUE(d.V >= 1, "logits must have at least one action");
        const int64_t k = logits.dim() - 1;
        rows.assign(logits.sizes().begin(), logits.sizes().end() - 1);
        d.n = 1;
        d.row_stride = d.V;
        // The leading dimensions must step through rows at one stride.
        bool first = true;
        for (int64_t i = k - 1; i >= 0; i--) {
            if (rows[i] != 1) {
                if (first) {
                    d.row_stride = logits.stride(i);
                } else {
                    TORCH_CHECK_VALUE(logits.stride(i) == d.row_stride * d.n || logits.numel() == 0,
                                      "the rows of logits must lie at one stride");
                }
                first = false;
            }
            d.n *= rows[i];
        }
        if (logits.numel() == 0) d.row_stride = d.V;
        TORCH_CHECK_VALUE(d.row_stride >= d.V, "the rows of logits must not overlap");
        need_sizes(action, "action", rows);
        need_contiguous(action, "action");
        switch (action.scalar_type()) {
            case at::kByte: d.action_dtype = GEAR_DTYPE_U8; break;
            case at::kInt: d.action_dtype = GEAR_DTYPE_I32; break;
            case at::kLong: d.action_dtype = GEAR_DTYPE_I64; break;
            default: TORCH_CHECK_VALUE(false, "action must be uint8, int32 or int64, not ", action.scalar_type());
        }
        mask = optional_of(o_mask, "mask", Kind::kFlags, dev);
        need_contiguous(mask, "mask");
        d.mask_group = mask.defined() ? group_of(mask, "mask") : 1;
        d.adv_group = d.weight_group = 1;
        d.d_action = action.data_ptr();
        d.d_mask = data<uint8_t>(mask);
    }
    at::Tensor per_row(PyObject* o, const char* name) const {
        const at::Tensor t = optional_of(o, name, Kind::kFloat, dev);
        if (t.defined()) need_sizes(t, name, rows);
        need_contiguous(t, name);
        return t;
    }
};

// policy_loss(logits, action, old_logp, adv, ref_logp, weight, mask, clip_low, clip_high, kl, entropy, denom,
//             grad, grad_scale, grad_loss, in_place, stream): (loss, logp, entropy, stats, grad or None)
PyObject* py_policy_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 17, [&]() -> PyObject* {
        Policy p(a[0], a[1], a[6]);
        const at::Tensor old_logp = p.per_row(a[2], "old_logp"), ref_logp = p.per_row(a[4], "ref_logp");
        TORCH_CHECK_VALUE(old_logp.defined(), "old_logp is missing");
        const at::Tensor adv = optional_of(a[3], "adv", Kind::kFloat, p.dev);
        TORCH_CHECK_VALUE(adv.defined(), "adv is missing");
        need_contiguous(adv, "adv");
        p.d.adv_group = p.group_of(adv, "adv");
        const at::Tensor weight = optional_of(a[5], "weight", Kind::kFloat, p.dev);
        need_contiguous(weight, "weight");
        if (weight.defined()) p.d.weight_group = p.group_of(weight, "weight");
        p.d.clip_low = as_float(a[7]);
        p.d.clip_high = as_float(a[8]);
        p.d.kl = as_float(a[9]);
        p.d.entropy = as_float(a[10]);
        p.d.denom = a[11] == Py_None ? 0.0f : as_float(a[11]);
        TORCH_CHECK_VALUE(a[11] == Py_None || p.d.denom > 0.0f, "denom must be above 0");
        const bool want_grad = as_bool(a[12]), in_place = as_bool(a[15]);
        p.d.grad_scale = as_float(a[13]);
        const at::Tensor grad_loss = optional_of(a[14], "grad_loss", Kind::kFloat, p.dev);
        TORCH_CHECK_VALUE(!grad_loss.defined() || grad_loss.numel() == 1, "grad_loss must hold one value");
        TORCH_CHECK_VALUE(!in_place || p.logits.is_contiguous(), "logits must be contiguous to be overwritten");
        void* s = as_ptr(a[16]);
        const c10::DeviceGuard guard(p.dev);
        int64_t work_bytes = 0;
        int rc = f_policy_sizes(&p.d, &work_bytes);
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        at::Tensor loss = make({}, at::kFloat, p.dev), stats = make({4}, at::kFloat, p.dev);
        at::Tensor logp = make(p.rows, at::kFloat, p.dev), entropy = make(p.rows, at::kFloat, p.dev), grad;
        if (want_grad) grad = in_place ? p.logits : make(p.logits.sizes(), p.logits.scalar_type(), p.dev);
        const at::Tensor work = workspace(work_bytes, p.dev);
        if (want_grad && in_place) {
            need_apart(p.logits, "logits", p.action, "action");
            need_apart(p.logits, "logits", p.mask, "mask");
            need_apart(p.logits, "logits", old_logp, "old_logp");
            need_apart(p.logits, "logits", ref_logp, "ref_logp");
            need_apart(p.logits, "logits", adv, "adv");
            need_apart(p.logits, "logits", weight, "weight");
            need_apart(p.logits, "logits", grad_loss, "grad_loss");
            overwrites(p.logits);
        }
        rc = without_gil([&] {
            return f_policy_loss(&p.d, p.logits.data_ptr(), data<float>(old_logp), data<float>(ref_logp), data<float>(adv),
                                 data<float>(weight), data<float>(grad_loss), data<float>(loss), data<float>(stats),
                                 data<float>(logp), data<float>(entropy), data<void>(grad), data<void>(work), work_bytes,
                                 s);
        });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        Tuple t(5);
        t.set(0, wrap(std::move(loss)));
        t.set(1, wrap(std::move(logp)));
        t.set(2, wrap(std::move(entropy)));
        t.set(3, wrap(std::move(stats)));
        if (want_grad) t.set(4, wrap(std::move(grad)));
        else t.none(4);
        return t.release();
    });
}

// action_logp(logits, action, mask, stream): (logp, entropy)
PyObject* py_action_logp(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return entry(n, 4, [&]() -> PyObject* {
        const Policy p(a[0], a[1], a[2]);
        void* s = as_ptr(a[3]);
        const c10::DeviceGuard guard(p.dev);
        at::Tensor logp = make(p.rows, at::kFloat, p.dev), entropy = make(p.rows, at::kFloat, p.dev);
        const int rc = without_gil([&] {
            return f_action_logp(&p.d, p.logits.data_ptr(), data<float>(logp), data<float>(entropy), s);
        });
        if (rc != GEAR_OK) return PyLong_FromLong(rc);
        Tuple t(2);
        t.set(0, wrap(std::move(logp)));
        t.set(1, wrap(std::move(entropy)));
        return t.release();
    });
}

#define GEAR_METHOD(name, doc) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(py_##name)), METH_FASTCALL, doc}
PyMethodDef methods[] = {
    GEAR_METHOD(bind, "addresses of the library's entry points"),
    GEAR_METHOD(plan, "column plan of a table"),
    GEAR_METHOD(select, "gear_select with allocated outputs"),
    GEAR_METHOD(collect, "gear_collect with allocated batches"),
    GEAR_METHOD(select_collect, "gear_select_collect with allocated outputs"),
    GEAR_METHOD(update, "gear_update_priorities"),
    GEAR_METHOD(select_shard, "gear_select_shard with allocated outputs"),
    GEAR_METHOD(is_weights, "gear_is_weights with allocated output"),
    GEAR_METHOD(topk_merge, "gear_topk_merge with allocated outputs"),
    GEAR_METHOD(recurrence, "gear_recurrence with allocated outputs"),
    GEAR_METHOD(recurrence_step, "gear_recurrence of one step"),
    GEAR_METHOD(recurrence_backward, "gear_recurrence_backward with allocated gradients"),
    GEAR_METHOD(advantages, "gear_advantages with allocated outputs"),
    GEAR_METHOD(policy_loss, "gear_policy_loss with allocated outputs"),
    GEAR_METHOD(action_logp, "gear_action_logp with allocated outputs"),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "Per-step calls of the experience-replay library.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding(void) { return PyModule_Create(&module); }

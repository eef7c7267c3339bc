// The C entry points as Python functions of tensors, and the allocation of results.
//
// What bounds it: a small call (one layer of 24 tokens, an update of a million weights) is 3 to 6 us on the GPU, and a
// program that issues them one after the other was bound by what the host did per call: through ctypes 6.6 us for a planned
// layer (2.5 of it the launch), 1.8 of them torch.empty from Python, 0.2 per tensor for its checks and 1 for the
// conversion of the arguments.  Here the conversions are made by the signature of the C function at compile time.
// Host time of a call: bsp_linear_planned 6.6 -> 4.9 us, an encoder layer's four 26.8 -> 20.0 (the GPU's part is 21.6),
// factors and update of 1024 x 1024 weights 12.6 -> 9.7, the layer in single precision 8.2 -> 5.3.
//
// The checks are the binding's own: a tensor is contiguous and on the GPU, and of its pointer's type where that function
// asks for it.  Only plain tensors are read directly; anything else is asked through its Python attributes, as before.
// The interpreter lock is released during the call, as ctypes does, and while results are allocated, as torch does.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <tuple>
#include <type_traits>
#include <utility>
#include <vector>

#include "bsp.h"

namespace {

enum Check : unsigned { kNone = 0, kFloat = 1, kByte = 2, kInt = 4, kAll = 7 };

bool wrong_place() {
    PyErr_SetString(PyExc_ValueError, "tensor must be a contiguous GPU tensor");
    return false;
}

bool wrong_type(PyObject *o, const char *want) {
    PyObject *dtype = PyObject_GetAttrString(o, "dtype");
    if (!dtype) return false;
    PyErr_Format(PyExc_ValueError, "expected dtype torch.%s, got %S", want, dtype);
    Py_DECREF(dtype);
    return false;
}

// An object that is no plain tensor: by its attributes.
bool read_other(PyObject *o, const char *want, void *&out) {
    PyObject *flag = PyObject_GetAttrString(o, "is_cuda");
    if (!flag) return false;
    const int cuda = PyObject_IsTrue(flag);
    Py_DECREF(flag);
    if (cuda < 0) return false;
    if (!cuda) return wrong_place();
    PyObject *dense = PyObject_CallMethod(o, "is_contiguous", nullptr);
    if (!dense) return false;
    const int contiguous = PyObject_IsTrue(dense);
    Py_DECREF(dense);
    if (contiguous < 0) return false;
    if (!contiguous) return wrong_place();
    if (want) {
        PyObject *dtype = PyObject_GetAttrString(o, "dtype");
        if (!dtype) return false;
        PyObject *name = PyObject_Str(dtype);
        Py_DECREF(dtype);
        if (!name) return false;
        const char *text = PyUnicode_AsUTF8(name);
        const bool same = text && strncmp(text, "torch.", 6) == 0 && strcmp(text + 6, want) == 0;
        Py_DECREF(name);
        if (!same) return PyErr_Occurred() ? false : wrong_type(o, want);
    }
    PyObject *at = PyObject_CallMethod(o, "data_ptr", nullptr);
    if (!at) return false;
    out = PyLong_AsVoidPtr(at);
    Py_DECREF(at);
    return !PyErr_Occurred();
}

bool read_tensor(PyObject *o, const char *want, at::ScalarType type, void *&out) {
    if (o == Py_None) {
        out = nullptr;
        return true;
    }
    if (!THPVariable_CheckExact(o)) return read_other(o, want, out);
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) return wrong_place();
    if (want && t.scalar_type() != type) return wrong_type(o, want);
    out = t.data_ptr();
    return true;
}

// What else stands for a number, as for ctypes: its own scalar of the argument's type, and an object that names another as its
// _as_parameter_.  A new reference, or null with the error that was set.
PyObject *other_number(PyObject *o, const char *scalar) {
    if (!PyErr_ExceptionMatches(PyExc_TypeError)) return nullptr;
    PyObject *type, *value, *trace;
    PyErr_Fetch(&type, &value, &trace);
    PyObject *n = strcmp(Py_TYPE(o)->tp_name, scalar) == 0 ? PyObject_GetAttrString(o, "value") : nullptr;
    if (!n) {
        PyErr_Clear();
        n = PyObject_GetAttrString(o, "_as_parameter_");
    }
    if (n) {
        Py_XDECREF(type);
        Py_XDECREF(value);
        Py_XDECREF(trace);
    } else {
        PyErr_Clear();
        PyErr_Restore(type, value, trace);
    }
    return n;
}

// The number that stands in another's place, which may name one in turn (without end, if it names itself).  Takes the reference.
template <typename T>
bool read_instead(PyObject *n, bool (*read_number)(PyObject *, T &), T &out) {
    bool ok = Py_EnterRecursiveCall(" while processing _as_parameter_") == 0;
    if (ok) {
        ok = read_number(n, out);
        Py_LeaveRecursiveCall();
    }
    Py_DECREF(n);
    return ok;
}

// Whole numbers: everything with __index__ (numpy's, a tensor of one).  Of one larger than the type the low bits.
template <typename T>
bool read_whole(PyObject *o, T &out) {
    PyObject *n = PyNumber_Index(o);
    if (!n) {
        n = other_number(o, std::is_unsigned_v<T> ? "c_ulong" : (sizeof(T) == 8 ? "c_long" : "c_int"));
        return n && read_instead(n, read_whole<T>, out);
    }
    out = static_cast<T>(PyLong_AsUnsignedLongLongMask(n));
    Py_DECREF(n);
    return true;
}

template <typename T>
bool read_real(PyObject *o, T &out) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyObject *n = other_number(o, std::is_same_v<T, float> ? "c_float" : "c_double");
        return n && read_instead(n, read_real<T>, out);
    }
    out = static_cast<T>(v);
    return true;
}

// STREAM: the argument is the stream, an address.
template <unsigned C, bool STREAM, typename T>
bool read(PyObject *o, T &out) {
    if constexpr (STREAM) {
        out = PyLong_AsVoidPtr(o);
        return !PyErr_Occurred();
    } else if constexpr (std::is_pointer_v<T>) {
        using V = std::remove_cv_t<std::remove_pointer_t<T>>;
        void *p = nullptr;
        bool ok;
        if constexpr (std::is_same_v<V, float> && (C & kFloat)) ok = read_tensor(o, "float32", at::kFloat, p);
        else if constexpr (std::is_same_v<V, uint8_t> && (C & kByte)) ok = read_tensor(o, "uint8", at::kByte, p);
        else if constexpr (std::is_same_v<V, int32_t> && (C & kInt)) ok = read_tensor(o, "int32", at::kInt, p);
        else ok = read_tensor(o, nullptr, at::kByte, p);
        out = static_cast<T>(p);
        return ok;
    } else if constexpr (std::is_floating_point_v<T>) {
        return read_real(o, out);
    } else {
        return read_whole(o, out);
    }
}

struct Unlocked {  // the interpreter lock, given up for its lifetime
    PyThreadState *state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

template <auto Fn, unsigned C>
struct Entry;
template <typename Ret, typename... A, Ret (*Fn)(A...), unsigned C>
struct Entry<Fn, C> {
    template <size_t... I>
    static PyObject *call(PyObject *const *args, std::index_sequence<I...>) {
        std::tuple<A...> a{};
        constexpr auto is_stream = [](size_t i) { return i == sizeof...(A) - 1; };
        if (!(read<C, is_stream(I) && std::is_pointer_v<A>>(args[I], std::get<I>(a)) && ...)) return nullptr;
        Ret r;
        {
            const Unlocked unlocked;
            r = Fn(std::get<I>(a)...);
        }
        if constexpr (std::is_signed_v<Ret>) return PyLong_FromLongLong(r);
        else return PyLong_FromUnsignedLongLong(r);
    }
    static PyObject *run(PyObject *, PyObject *const *args, Py_ssize_t n) {
        HANDLE_TH_ERRORS
        if (n != (Py_ssize_t)sizeof...(A)) {
            PyErr_Format(PyExc_TypeError, "this function takes %d arguments (%zd given)", (int)sizeof...(A), n);
            return nullptr;
        }
        return call(args, std::make_index_sequence<sizeof...(A)>{});
        END_HANDLE_TH_ERRORS
    }
};

// empty() beside an object that is no plain tensor: torch.empty with the object's own device.
PyObject *empty_beside_other(PyObject *like, const char *type, const int64_t *size, int dims) {
    PyObject *torch = PyImport_ImportModule("torch");
    if (!torch) return nullptr;
    PyObject *make = PyObject_GetAttrString(torch, "empty"), *dtype = PyObject_GetAttrString(torch, type);
    PyObject *device = PyObject_GetAttrString(like, "device"), *result = nullptr;
    PyObject *args = dims == 1 ? Py_BuildValue("((L))", (long long)size[0]) : Py_BuildValue("((LL))", (long long)size[0], (long long)size[1]);
    if (make && dtype && device && args) {
        PyObject *named = Py_BuildValue("{s:O,s:O}", "dtype", dtype, "device", device);
        if (named) result = PyObject_Call(make, args, named);
        Py_XDECREF(named);
    }
    Py_DECREF(torch);
    Py_XDECREF(make);
    Py_XDECREF(dtype);
    Py_XDECREF(device);
    Py_XDECREF(args);
    return result;
}

// empty(like, type, n) or empty(like, type, n, m): a tensor on the device of `like`; type: a bsp_dtype, 3 uint8, 4 int32.
PyObject *empty(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 3 && n != 4) {
        PyErr_SetString(PyExc_TypeError, "empty(tensor, type, n[, m])");
        return nullptr;
    }
    constexpr at::ScalarType types[] = {at::kFloat, at::kBFloat16, at::kHalf, at::kByte, at::kInt};
    constexpr const char *names[] = {"float32", "bfloat16", "float16", "uint8", "int32"};
    const long long type = PyLong_AsLongLong(args[1]);
    int64_t size[2] = {0, 0};
    for (Py_ssize_t i = 2; i < n; ++i) size[i - 2] = PyLong_AsLongLong(args[i]);
    if (PyErr_Occurred()) return nullptr;
    if (type < 0 || type > 4) {
        PyErr_SetString(PyExc_ValueError, "unknown type");
        return nullptr;
    }
    if (!THPVariable_CheckExact(args[0])) return empty_beside_other(args[0], names[type], size, (int)n - 2);
    const auto options = at::TensorOptions().dtype(types[type]).device(THPVariable_Unpack(args[0]).device());
    at::Tensor t;
    {
        const Unlocked unlocked;  // (an allocation may wait for the device)
        t = at::empty(at::IntArrayRef(size, (size_t)(n - 2)), options);
    }
    return THPVariable_Wrap(std::move(t));
    END_HANDLE_TH_ERRORS
}

// last(tensor): the last element of a vector of whole numbers, read back; of an object that is no plain tensor int(o[-1].item()).
PyObject *last(PyObject *, PyObject *o) {
    HANDLE_TH_ERRORS
    if (!THPVariable_CheckExact(o)) {
        PyObject *at = PyLong_FromLong(-1), *element = at ? PyObject_GetItem(o, at) : nullptr;
        PyObject *value = element ? PyObject_CallMethod(element, "item", nullptr) : nullptr;
        PyObject *whole = value ? PyNumber_Long(value) : nullptr;
        Py_XDECREF(at);
        Py_XDECREF(element);
        Py_XDECREF(value);
        return whole;
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    int64_t v;
    {
        const Unlocked unlocked;
        v = t.select(0, -1).item().toLong();
    }
    return PyLong_FromLongLong(v);
    END_HANDLE_TH_ERRORS
}

// ---- lists of tensors -----------------------------------------------------------------------------------------------------------
struct Owned {  // a reference that ends with its scope
    PyObject *o;
    ~Owned() { Py_XDECREF(o); }
};

PyObject *bad_list(const char *what) {
    PyErr_Format(PyExc_ValueError, "bsp_adamw_step: %s", what);
    return nullptr;
}

// A plain contiguous tensor on device `device`; null with the error set.
const at::Tensor *listed_tensor(PyObject *o, const char *name, int64_t device) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "bsp_adamw_step: %s must hold tensors, got %s", name, Py_TYPE(o)->tp_name);
        return nullptr;
    }
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous() || t.device().index() != device) {
        PyErr_Format(PyExc_ValueError, "bsp_adamw_step: %s must hold contiguous tensors on the current device", name);
        return nullptr;
    }
    return &t;
}

// bsp_adamw_step(W, G, m, v, scales, copies, keep, alpha, R, weight_decay, bits, lam, lr, beta1, beta2, eps, t, seed, lr_t, grad_scale,
// device, stream): the lists' tensors as descriptions.  (A model's 400 tensors one by one from Python would take ten times as long as their step.)
PyObject *adamw_step(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (n_args != 22) {
        PyErr_Format(PyExc_TypeError, "this function takes 22 arguments (%zd given)", n_args);
        return nullptr;
    }
    constexpr const char *names[] = {"W", "G", "m", "v", "scales", "copies", "keep", "alpha"};
    PyObject *list[8];
    Owned owned[10] = {};
    Py_ssize_t count = -1;
    for (int i = 0; i < 8; ++i) {
        list[i] = nullptr;
        if (args[i] == Py_None && i >= 4) continue;
        list[i] = owned[i].o = PySequence_Fast(args[i], "bsp_adamw_step takes lists of tensors");
        if (!list[i]) return nullptr;
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(list[i]);
        if (count < 0) count = n;
        if (n != count) return bad_list("the lists must have one length");
    }
    PyObject *rows = nullptr, *decays = nullptr;  // lists, or numbers for all tensors
    int32_t row = 0;
    float decay = 0.0f;
    if (PyList_Check(args[8]) || PyTuple_Check(args[8])) rows = owned[8].o = PySequence_Fast(args[8], "");
    else if (!read_whole(args[8], row)) return nullptr;
    if (PyList_Check(args[9]) || PyTuple_Check(args[9])) decays = owned[9].o = PySequence_Fast(args[9], "");
    else if (!read_real(args[9], decay)) return nullptr;
    for (PyObject *l : {rows, decays})
        if (l && PySequence_Fast_GET_SIZE(l) != count) return bad_list("the lists must have one length");
    int bits;
    double real[5];
    int64_t t, device;
    uint64_t seed;
    void *lr_t, *grad_scale, *stream;
    if (!read_whole(args[10], bits)) return nullptr;
    for (int i = 0; i < 5; ++i)
        if (!read_real(args[11 + i], real[i])) return nullptr;
    if (!read_whole(args[16], t) || !read_whole(args[17], seed) || !read_tensor(args[18], "float32", at::kFloat, lr_t) ||
        !read_tensor(args[19], "float32", at::kFloat, grad_scale) || !read_whole(args[20], device))
        return nullptr;
    for (int i = 18; i < 20; ++i)
        if (args[i] != Py_None && THPVariable_Check(args[i])) {
            const at::Tensor &x = THPVariable_Unpack(args[i]);
            if (x.device().index() != device || x.numel() < (i == 18 ? 2 : 1)) return bad_list("lr_t holds 2 and grad_scale 1 number on the current device");
        }
    stream = PyLong_AsVoidPtr(args[21]);
    if (PyErr_Occurred()) return nullptr;

    std::vector<bsp_adamw_tensor> tensors((size_t)count);
    at::ScalarType gdt = at::kFloat, cdt = at::kBFloat16;
    bool copies = false;
    const at::ScalarType moment = bits == 8 ? at::kFloat8_e4m3fn : at::kFloat;
    for (Py_ssize_t i = 0; i < count; ++i) {
        const at::Tensor *x[8];
        for (int k = 0; k < 8; ++k) {
            PyObject *o = list[k] ? PySequence_Fast_GET_ITEM(list[k], i) : Py_None;
            if (o == Py_None && k >= 5) {
                x[k] = nullptr;
                continue;
            }
            if (k == 4 && !list[4]) {
                x[4] = nullptr;
                continue;
            }
            x[k] = listed_tensor(o, names[k], device);
            if (!x[k]) return nullptr;
        }
        const at::Tensor &w = *x[0];
        if (w.scalar_type() != at::kFloat) return bad_list("W must be float32");
        if (i == 0) gdt = x[1]->scalar_type();
        if (gdt != at::kFloat && gdt != at::kBFloat16 && gdt != at::kHalf) return bad_list("G must be float32, bfloat16 or float16");
        if (x[1]->scalar_type() != gdt || x[1]->sizes() != w.sizes()) return bad_list("G must have the shapes of W and one dtype");
        for (int k = 2; k < 4; ++k)
            if (x[k]->scalar_type() != moment || x[k]->sizes() != w.sizes())
                return bad_list("m and v must have the shapes of W and be float32, or float8_e4m3fn with scales");
        bsp_adamw_tensor &d = tensors[(size_t)i];
        const int64_t n = w.numel();
        const bool grouped = x[6] || x[7];
        d.N = grouped && w.dim() > 0 ? w.size(-1) : 1;  // (without groups the shape is of no account)
        d.M = d.N ? n / d.N : 0;
        d.R = row;
        d.weight_decay = decay;
        if (rows && !read_whole(PySequence_Fast_GET_ITEM(rows, i), d.R)) return nullptr;
        if (decays && !read_real(PySequence_Fast_GET_ITEM(decays, i), d.weight_decay)) return nullptr;
        if (x[4] && (x[4]->scalar_type() != at::kFloat || x[4]->numel() != 2 * ((n + 255) / 256))) return bad_list("scales must be float32, 2 for every 256 elements");
        if (x[5]) {
            if (!copies) cdt = x[5]->scalar_type();
            copies = true;
            if (x[5]->scalar_type() != cdt || (cdt != at::kBFloat16 && cdt != at::kHalf) || x[5]->sizes() != w.sizes())
                return bad_list("copies must have the shapes of W and one 16-bit dtype");
        }
        if (grouped && n && (d.R <= 0 || d.M % d.R != 0)) return bad_list("a tensor with keep or alpha must have whole row-blocks of R rows");
        if (x[6] && (x[6]->scalar_type() != at::kByte || (n && x[6]->numel() != n / d.R))) return bad_list("keep must be uint8 [M / R, N]");
        if (x[7] && (x[7]->scalar_type() != at::kFloat || (n && x[7]->numel() != n / d.R))) return bad_list("alpha must be float32 [M / R, N]");
        void *at[8];
        for (int k = 0; k < 8; ++k) at[k] = x[k] ? x[k]->data_ptr() : nullptr;
        d.w = (float *)at[0];
        d.g = at[1];
        d.m = at[2];
        d.v = at[3];
        d.scales = (float *)at[4];
        d.copy = at[5];
        d.keep = (const uint8_t *)at[6];
        d.alpha = (const float *)at[7];
    }
    int st;
    {
        const Unlocked unlocked;
        st = bsp_adamw_step(tensors.data(), count, gdt == at::kFloat ? BSP_F32 : (gdt == at::kBFloat16 ? BSP_BF16 : BSP_F16),
                            cdt == at::kHalf ? BSP_F16 : BSP_BF16, bits, real[0], real[1], real[2], real[3], real[4], t, (uint32_t)seed,
                            (const float *)lr_t, (const float *)grad_scale, stream);
    }
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// ---- calls with their checks and results ----------------------------------------------------------------------------------------------------
// Checks, results and the call in one function.  One by one from Python the twelve tensors and seven results of a norm's backward pass took 16 us,
// its kernels 9; a layer of one token in 8 bits 6.5, its kernel 4.
struct RowArgs {
    const char *where;
    int64_t device;
    const at::Tensor *like = nullptr;

    bool fail(const char *what) const {
        PyErr_Format(PyExc_ValueError, "%s: %s", where, what);
        return false;
    }
    // A contiguous tensor on the current device, or none.
    bool take(PyObject *o, const at::Tensor *&t) const {
        t = nullptr;
        if (o == Py_None) return true;
        if (!THPVariable_Check(o)) {
            PyErr_Format(PyExc_TypeError, "%s takes tensors, got %s", where, Py_TYPE(o)->tp_name);
            return false;
        }
        t = &THPVariable_Unpack(o);
        return t->is_cuda() && t->is_contiguous() && t->device().index() == device ? true : fail("tensors must be contiguous and on the current device");
    }
    bool rows(PyObject *o, const at::Tensor *&t) {  // [T, H] of one shape and type, the first one's
        if (!take(o, t)) return false;
        if (!t) return true;
        if (!like) {
            if (t->dim() != 2 || (t->scalar_type() != at::kFloat && t->scalar_type() != at::kBFloat16 && t->scalar_type() != at::kHalf))
                return fail("rows must be [T, H] of float32, bfloat16 or float16");
            like = t;
        }
        return t->scalar_type() == like->scalar_type() && t->sizes() == like->sizes() ? true : fail("the [T, H] tensors must share one shape and dtype");
    }
    bool vector(PyObject *o, const at::Tensor *&t) const {
        if (!take(o, t)) return false;
        return !t || (t->scalar_type() == like->scalar_type() && t->numel() == like->size(1)) ? true
                                                                                               : fail("weights and biases must have H elements of the dtype of the rows");
    }
    bool gate(PyObject *o, const at::Tensor *&t, int64_t &gate_rows) const {
        gate_rows = 0;
        if (!take(o, t) || !t) return !PyErr_Occurred();
        if (t->scalar_type() != like->scalar_type() || (t->dim() != 1 && t->dim() != 2) || t->size(-1) != like->size(1))
            return fail("gate must be [gate_rows, H] of the dtype of the rows");
        gate_rows = t->dim() == 1 ? 1 : t->size(0);
        return true;
    }
    bool stats(PyObject *o, const at::Tensor *&t) const {
        if (!take(o, t)) return false;
        return !t || (t->scalar_type() == at::kFloat && t->dim() == 2 && t->size(0) == like->size(0) && t->size(1) == 2) ? true
                                                                                                                            : fail("stats must be float32 [T, 2]");
    }
    int type() const { return like->scalar_type() == at::kFloat ? BSP_F32 : (like->scalar_type() == at::kBFloat16 ? BSP_BF16 : BSP_F16); }
    // (what at::empty comes to on a GPU, without its way there)
    at::Tensor make(at::IntArrayRef size, at::ScalarType t) const { return at::Tensor(at::detail::empty_cuda(size, t, like->device(), c10::nullopt)); }
};

void *address(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }

// (status, results...): a defined tensor as it is, else None.
PyObject *with_status(int st, at::Tensor *results, int n) {
    PyObject *all = PyTuple_New(n + 1);
    if (!all) return nullptr;
    PyTuple_SET_ITEM(all, 0, PyLong_FromLong(st));
    for (int i = 0; i < n; ++i) PyTuple_SET_ITEM(all, i + 1, THPVariable_Wrap(results[i]));  // (None for an undefined one)
    return all;
}

// A quantised matrix [rows, cols] given as codes and scales.
struct Coded {
    const at::Tensor *codes, *scales;
    int64_t rows, cols;
    int layout;
    // args: codes, scales, rows, cols, layout
    bool read(const RowArgs &a, PyObject *const *args) {
        if (!a.take(args[0], codes) || !a.take(args[1], scales) || !read_whole(args[2], rows) || !read_whole(args[3], cols) || !read_whole(args[4], layout))
            return false;
        const int64_t steps = (cols + 127) / 128, lines = layout == BSP_FP8_BLOCK ? (rows + 127) / 128 : rows;
        return codes && scales && rows >= 0 && cols > 0 && codes->scalar_type() == at::kFloat8_e4m3fn && codes->numel() == rows * steps * 128 &&
                       scales->scalar_type() == at::kByte && scales->numel() == lines * steps
                   ? true
                   : a.fail("codes (float8_e4m3fn) and scales (uint8) do not have the sizes of their matrix");
    }
};

// fp8_quant(X, layout, want, device, stream) -> (status, Q, S, Qt, St); want: 1 for X, 2 for the transposed X
PyObject *fp8_quant(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (n_args != 5) {
        PyErr_Format(PyExc_TypeError, "this function takes 5 arguments (%zd given)", n_args);
        return nullptr;
    }
    RowArgs a{"bsp_fp8_quant", 0};
    const at::Tensor *X;
    int layout;
    uint32_t want;
    if (!read_whole(args[3], a.device) || !a.rows(args[0], X)) return nullptr;
    if (!X) return a.fail("X must be a tensor"), nullptr;
    if (!read_whole(args[1], layout) || !read_whole(args[2], want)) return nullptr;
    void *stream = PyLong_AsVoidPtr(args[4]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out[4];
    int st;
    {
        const Unlocked unlocked;
        const int64_t rows = X->size(0), cols = X->size(1);
        for (int i = 0; i < 2; ++i)
            if ((want >> i) & 1u) {
                const int64_t r = i ? cols : rows, steps = ((i ? rows : cols) + 127) / 128;
                out[2 * i] = a.make({r, 128 * steps}, at::kFloat8_e4m3fn);
                out[2 * i + 1] = a.make({layout == BSP_FP8_BLOCK ? (r + 127) / 128 : r, steps}, at::kByte);
            }
        auto at_of = [](at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
        st = bsp_fp8_quant(X->data_ptr(), a.type(), rows, cols, layout, at_of(out[0]), (uint8_t *)at_of(out[1]), at_of(out[2]), (uint8_t *)at_of(out[3]), stream);
    }
    return with_status(st, out, 4);
    END_HANDLE_TH_ERRORS
}

// matmul_fp8(A's codes, scales, rows, cols, layout, B's, bias, act, residual, type, Y, ws, device, stream) -> (status, Y); type: a bsp_dtype, of Y where that is None
PyObject *matmul_fp8(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (n_args != 18) {
        PyErr_Format(PyExc_TypeError, "this function takes 18 arguments (%zd given)", n_args);
        return nullptr;
    }
    RowArgs a{"bsp_matmul_fp8", 0};
    Coded A, B;
    const at::Tensor *bias, *residual, *Y, *ws;
    int act, type;
    if (!read_whole(args[16], a.device) || !A.read(a, args) || !B.read(a, args + 5) || !a.take(args[10], bias) || !read_whole(args[11], act) ||
        !a.take(args[12], residual) || !read_whole(args[13], type) || !a.take(args[14], Y) || !a.take(args[15], ws))
        return nullptr;
    void *stream = PyLong_AsVoidPtr(args[17]);
    if (PyErr_Occurred()) return nullptr;
    if (A.layout != BSP_FP8_ROW || A.cols != B.cols) return a.fail("A must be quantised by rows and have the columns of B"), nullptr;
    constexpr at::ScalarType types[] = {at::kFloat, at::kBFloat16, at::kHalf};
    if (type < 0 || type > 2) return a.fail("unknown type"), nullptr;
    const int64_t T = A.rows, M = B.rows, K = A.cols;
    if (bias && (bias->scalar_type() != types[type] || bias->numel() != M)) return a.fail("bias must have M elements of the dtype of the result"), nullptr;
    for (const at::Tensor *t : {residual, Y})
        if (t && (t->scalar_type() != types[type] || t->dim() != 2 || t->size(0) != T || t->size(1) != M))
            return a.fail("residual and Y must be [T, M] tensors of the dtype of the result"), nullptr;
    a.like = A.codes;
    at::Tensor out;
    int st;
    {
        const Unlocked unlocked;
        out = Y ? *Y : a.make({T, M}, types[type]);
        at::Tensor scratch;
        const size_t bytes = ws ? (size_t)ws->nbytes() : bsp_matmul_fp8_workspace_bytes(T, M, K);
        if (!ws && bytes) scratch = a.make({(int64_t)bytes}, at::kByte);
        st = bsp_matmul_fp8(A.codes->data_ptr(), (const uint8_t *)A.scales->data_ptr(), B.codes->data_ptr(), (const uint8_t *)B.scales->data_ptr(), B.layout,
                            T, M, K, address(bias), act, address(residual), out.data_ptr(), type, !bytes ? nullptr : ws ? ws->data_ptr() : scratch.data_ptr(), bytes, stream);
    }
    return with_status(st, &out, 1);
    END_HANDLE_TH_ERRORS
}

// linear_fp8(X, codes, scales, rows, cols, layout, bias, act, residual, Y, ws, device, stream) -> (status, Y)
PyObject *linear_fp8(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (n_args != 13) {
        PyErr_Format(PyExc_TypeError, "this function takes 13 arguments (%zd given)", n_args);
        return nullptr;
    }
    RowArgs a{"bsp_linear_fp8", 0};
    const at::Tensor *X, *bias, *residual, *Y, *ws;
    Coded W;
    int act;
    if (!read_whole(args[11], a.device) || !a.rows(args[0], X)) return nullptr;
    if (!X) return a.fail("X must be a tensor"), nullptr;
    if (!W.read(a, args + 1) || !a.take(args[6], bias) || !read_whole(args[7], act) || !a.take(args[8], residual) || !a.take(args[9], Y) ||
        !a.take(args[10], ws))
        return nullptr;
    void *stream = PyLong_AsVoidPtr(args[12]);
    if (PyErr_Occurred()) return nullptr;
    const int64_t T = X->size(0), M = W.rows, N = W.cols;
    if (X->size(1) != N) return a.fail("X has the wrong number of columns"), nullptr;
    const at::ScalarType type = X->scalar_type();
    if (bias && (bias->scalar_type() != type || bias->numel() != M)) return a.fail("bias must have M elements of the dtype of X"), nullptr;
    for (const at::Tensor *t : {residual, Y})
        if (t && (t->scalar_type() != type || t->dim() != 2 || t->size(0) != T || t->size(1) != M))
            return a.fail("residual and Y must be [T, M] tensors of the dtype of X"), nullptr;
    at::Tensor out;
    int st;
    {
        const Unlocked unlocked;
        out = Y ? *Y : a.make({T, M}, type);
        at::Tensor scratch;
        size_t bytes = ws ? (size_t)ws->nbytes() : bsp_linear_fp8_workspace_bytes(T, M, N);
        if (!ws && bytes) scratch = a.make({(int64_t)bytes}, at::kByte);
        st = bsp_linear_fp8(X->data_ptr(), a.type(), T, M, N, W.codes->data_ptr(), (const uint8_t *)W.scales->data_ptr(), W.layout, address(bias), act,
                            address(residual), out.data_ptr(), ws ? ws->data_ptr() : (bytes ? scratch.data_ptr() : nullptr), bytes, stream);
    }
    return with_status(st, &out, 1);
    END_HANDLE_TH_ERRORS
}

enum NormWant : unsigned { kWantZ = 1, kWantStatsPost = 2, kWantStatsPre = 4 };

// block_norm(X, F, norms, kind, eps, x_scale, gate, w_post, b_post, w_pre, b_pre, Z, H, want, device, stream) -> (status, Z, H, stats_post, stats_pre)
PyObject *block_norm(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (n_args != 16) {
        PyErr_Format(PyExc_TypeError, "this function takes 16 arguments (%zd given)", n_args);
        return nullptr;
    }
    RowArgs a{"bsp_block_norm", 0};
    const at::Tensor *X, *F, *gate, *w[4], *Z, *H;
    int norms, kind;
    float eps, x_scale;
    int64_t gate_rows;
    uint32_t want;
    if (!read_whole(args[14], a.device) || !a.rows(args[0], X)) return nullptr;
    if (!X) return a.fail("X must be a tensor"), nullptr;
    if (!a.rows(args[1], F) || !read_whole(args[2], norms) || !read_whole(args[3], kind) || !read_real(args[4], eps) || !read_real(args[5], x_scale) ||
        !a.gate(args[6], gate, gate_rows) || !a.rows(args[11], Z) || !a.rows(args[12], H) || !read_whole(args[13], want))
        return nullptr;
    for (int i = 0; i < 4; ++i)
        if (!a.vector(args[7 + i], w[i])) return nullptr;
    void *stream = PyLong_AsVoidPtr(args[15]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out[4];
    int st;
    {
        const Unlocked unlocked;
        const int64_t T = X->size(0), width = X->size(1);
        const bool pre = norms & BSP_NORM_PRE;
        if (Z) out[0] = *Z;
        else if ((want & kWantZ) || !pre) out[0] = a.make({T, width}, X->scalar_type());
        if (H) out[1] = *H;
        else if (pre) out[1] = a.make({T, width}, X->scalar_type());
        if ((norms & BSP_NORM_POST) && (want & kWantStatsPost)) out[2] = a.make({T, 2}, at::kFloat);
        if (pre && (want & kWantStatsPre)) out[3] = a.make({T, 2}, at::kFloat);
        auto at_of = [](at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
        st = bsp_block_norm(address(X), address(F), a.type(), T, width, norms, kind, eps, x_scale, address(gate), gate_rows, address(w[0]),
                            address(w[1]), address(w[2]), address(w[3]), at_of(out[0]), at_of(out[1]), (float *)at_of(out[2]), (float *)at_of(out[3]), stream);
    }
    return with_status(st, out, 4);
    END_HANDLE_TH_ERRORS
}

// block_norm_backward(dZ, dH, Z, F, norms, kind, x_scale, gate, w_post, b_post, w_pre, b_pre, stats_post, stats_pre, dX, dF, want, ws, device, stream)
// -> (status, dx, df, dw_post, db_post, dw_pre, db_pre, dgate); want: a bit for each of these in turn.
PyObject *block_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (n_args != 20) {
        PyErr_Format(PyExc_TypeError, "this function takes 20 arguments (%zd given)", n_args);
        return nullptr;
    }
    RowArgs a{"bsp_block_norm_backward", 0};
    const at::Tensor *dZ, *dH, *Z, *F, *gate, *w[4], *sp, *sq, *dX, *dF, *ws;
    int norms, kind;
    float x_scale;
    int64_t gate_rows;
    uint32_t want;
    if (!read_whole(args[18], a.device) || !a.rows(args[0], dZ) || !a.rows(args[1], dH)) return nullptr;
    if (!a.like) return a.fail("one of dZ and dH must be a tensor"), nullptr;
    if (!a.rows(args[2], Z) || !a.rows(args[3], F) || !read_whole(args[4], norms) || !read_whole(args[5], kind) || !read_real(args[6], x_scale) ||
        !a.gate(args[7], gate, gate_rows) || !a.stats(args[12], sp) || !a.stats(args[13], sq) || !a.rows(args[14], dX) || !a.rows(args[15], dF) ||
        !read_whole(args[16], want) || !a.take(args[17], ws))
        return nullptr;
    for (int i = 0; i < 4; ++i)
        if (!a.vector(args[8 + i], w[i])) return nullptr;
    void *stream = PyLong_AsVoidPtr(args[19]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out[7];
    int st;
    {
        const Unlocked unlocked;
        const int64_t T = a.like->size(0), H = a.like->size(1);
        const at::ScalarType type = a.like->scalar_type();
        const bool post = norms & BSP_NORM_POST, pre = norms & BSP_NORM_PRE;
        if (dX) out[0] = *dX;
        else if (want & 1u) out[0] = a.make({T, H}, type);
        if (dF) out[1] = *dF;
        else if (want & 2u) out[1] = a.make({T, H}, type);
        const bool there[4] = {post && w[0], post && w[1], pre && w[2], pre && w[3]};
        bool any = false;
        for (int i = 0; i < 4; ++i)
            if (there[i] && ((want >> (2 + i)) & 1u)) out[2 + i] = a.make({H}, at::kFloat), any = true;
        if (gate && (want & 64u)) out[6] = a.make({gate_rows, H}, at::kFloat), any = true;
        at::Tensor scratch;
        size_t bytes = ws ? (size_t)ws->nbytes() : 0;
        if (!ws && any) {
            bytes = bsp_block_norm_backward_workspace_bytes(T, H, gate_rows);
            scratch = a.make({(int64_t)bytes}, at::kByte);
        }
        auto at_of = [](at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
        st = bsp_block_norm_backward(address(dZ), address(dH), address(Z), address(F), a.type(), T, H, norms, kind, x_scale, address(gate), gate_rows,
                                     address(w[0]), address(w[1]), address(w[2]), (const float *)address(sp), (const float *)address(sq), at_of(out[0]),
                                     at_of(out[1]), (float *)at_of(out[2]), (float *)at_of(out[3]), (float *)at_of(out[4]), (float *)at_of(out[5]),
                                     (float *)at_of(out[6]), ws ? ws->data_ptr() : at_of(scratch), bytes, stream);
    }
    return with_status(st, out, 7);
    END_HANDLE_TH_ERRORS
}

#define BSP_ENTRY(name, check) \
    {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&Entry<&name, check>::run)), METH_FASTCALL, nullptr}

PyMethodDef methods[] = {
    BSP_ENTRY(bsp_group_norms, kFloat),
    BSP_ENTRY(bsp_group_norms_grad, kFloat),
    BSP_ENTRY(bsp_prune_mask, kFloat | kByte),
    BSP_ENTRY(bsp_prune_mask_workspace_bytes, kNone),
    BSP_ENTRY(bsp_prune_mask_count, kAll),
    BSP_ENTRY(bsp_pack_count, kAll),
    BSP_ENTRY(bsp_pack, kAll),
    BSP_ENTRY(bsp_mask_weights, kByte),
    BSP_ENTRY(bsp_adam_step, kFloat | kByte),
    BSP_ENTRY(bsp_linear_workspace_bytes, kNone),
    BSP_ENTRY(bsp_linear_sized, kNone),
    BSP_ENTRY(bsp_linear_transposed_workspace_bytes, kNone),
    BSP_ENTRY(bsp_linear_transposed_ws, kNone),
    BSP_ENTRY(bsp_linear_dvals_workspace_bytes, kNone),
    BSP_ENTRY(bsp_linear_dvals, kNone),
    BSP_ENTRY(bsp_linear_plan_bytes, kNone),
    BSP_ENTRY(bsp_linear_plan, kNone),
    BSP_ENTRY(bsp_linear_planned, kNone),
    BSP_ENTRY(bsp_linear_planned_fused, kNone),
    {"fp8_quant", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&fp8_quant)), METH_FASTCALL, nullptr},
    {"matmul_fp8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&matmul_fp8)), METH_FASTCALL, nullptr},
    {"linear_fp8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&linear_fp8)), METH_FASTCALL, nullptr},
    {"block_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&block_norm)), METH_FASTCALL, nullptr},
    {"block_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&block_norm_backward)), METH_FASTCALL, nullptr},
    {"bsp_adamw_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&adamw_step)), METH_FASTCALL, nullptr},
    {"empty", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&empty)), METH_FASTCALL, nullptr},
    {"last", last, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_bsp_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bsp_host() { return PyModule_Create(&module_def); }

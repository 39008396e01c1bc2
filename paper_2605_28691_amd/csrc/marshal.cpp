// The calls of the Python binding, marshalled natively: every entry point of include/skiparse.h that launches kernels as a function of a CPython
// module, with the argument list of the C function, tensors in the places of device pointers.
//
// A small call is bound by what it costs to issue it: a kernel of 3 us behind 5.2 us of host work.  Of these the native call takes 3.9, nearly all of it the
// launch (a fill of a tensor by torch, one launch as well, takes 4.0), the result's tensor 1.1 and the checks and look-ups in Python 0.5.  By way of ctypes, with
// an address asked for tensor by tensor in Python, the call took 2 us more.  Here an argument costs nanoseconds.
//
// Only plain arguments are taken: torch.Tensor itself, on the GPU and contiguous, int itself within the range of the C type, float itself.  With anything else, and to turn a
// code into an exception, the module calls the functions that the binding has given it, so that what those accept, refuse and raise does not
// depend on this module.
//
// The module is not linked to the library: the binding hands it the addresses in the copy that it has opened itself, so that a process that
// rebuilds the library calls one copy only.
#include <Python.h>
#include <ATen/DimVector.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cxxabi.h>

#include <climits>
#include <cstring>
#include <tuple>
#include <utility>

#include "../../include/skiparse.h"

namespace {

#ifndef BUILT_FOR
#error "the torch that the headers belong to"
#endif

PyObject* g_general = nullptr;  // (name, *arguments): the same call by way of ctypes
PyObject* g_failed = nullptr;   // (code, name): raises

template <typename T>
struct Arg;
template <>
struct Arg<int> {
    static bool get(PyObject* o, int& v) {
        if (!PyLong_CheckExact(o)) return false;
        int over;
        const long n = PyLong_AsLongAndOverflow(o, &over);
        v = (int)n;
        return over == 0 && v == n;
    }
};
template <>
struct Arg<unsigned> {
    static bool get(PyObject* o, unsigned& v) {
        if (!PyLong_CheckExact(o)) return false;
        int over;
        const long n = PyLong_AsLongAndOverflow(o, &over);
        v = (unsigned)n;
        return over == 0 && (long)v == n;
    }
};
template <>
struct Arg<size_t> {
    static bool get(PyObject* o, size_t& v) {
        if (!PyLong_CheckExact(o)) return false;
        int over;
        const long n = PyLong_AsLongAndOverflow(o, &over);
        v = (size_t)n;
        return over == 0 && n >= 0;
    }
};
template <>
struct Arg<float> {
    static bool get(PyObject* o, float& v) {
        if (!PyFloat_CheckExact(o)) return false;
        v = (float)PyFloat_AS_DOUBLE(o);
        return true;
    }
};
template <>
struct Arg<double> {
    static bool get(PyObject* o, double& v) {
        if (!PyFloat_CheckExact(o)) return false;
        v = PyFloat_AS_DOUBLE(o);
        return true;
    }
};
template <typename P>
struct Arg<P*> {
    static bool get(PyObject* o, P*& v) {
        if (!THPVariable_CheckExact(o)) return false;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) return false;
        v = (P*)t.data_ptr();
        return true;
    }
};

// Argument I of N: the last one is the stream's handle; the arguments in the set NONE, a bit each, may be None.
template <size_t I, size_t N, unsigned NONE, typename T>
bool get_arg(PyObject* o, T& v) {
    if constexpr (I + 1 == N) {
        if (!PyLong_CheckExact(o)) return false;
        v = (T)(uintptr_t)PyLong_AsUnsignedLongLongMask(o);
        return true;
    } else {
        if constexpr (NONE >> I & 1u) {
            if (o == Py_None) {
                v = nullptr;
                return true;
            }
        }
        return Arg<T>::get(o, v);
    }
}

// The arguments as they came, with one more in front.
PyObject* pass_on(PyObject* callable, PyObject* first, PyObject* const* args, Py_ssize_t n) {
    PyObject* all = PyTuple_New(n + 1);
    if (all == nullptr) return nullptr;
    Py_INCREF(first);
    PyTuple_SET_ITEM(all, 0, first);
    for (Py_ssize_t i = 0; i < n; i++) {
        Py_INCREF(args[i]);
        PyTuple_SET_ITEM(all, i + 1, args[i]);
    }
    PyObject* r = PyObject_CallObject(callable, all);
    Py_DECREF(all);
    return r;
}

PyObject* general(const char* name, PyObject* const* args, Py_ssize_t n) {
    if (g_general == nullptr) {
        PyErr_SetString(PyExc_RuntimeError, "the binding has not been set up");
        return nullptr;
    }
    PyObject* first = PyUnicode_FromString(name);
    if (first == nullptr) return nullptr;
    PyObject* r = pass_on(g_general, first, args, n);
    Py_DECREF(first);
    return r;
}

template <unsigned NONE, typename... A, size_t... I>
PyObject* call_with(int (*fn)(A...), const char* name, PyObject* const* args, Py_ssize_t n, std::index_sequence<I...>) {
    std::tuple<A...> v;
    bool plain = n == (Py_ssize_t)sizeof...(A) && g_general != nullptr && g_failed != nullptr;
    try {
        plain = plain && (get_arg<I, sizeof...(A), NONE>(args[I], std::get<I>(v)) && ...);
    } catch (...) {  // a tensor without storage: the general way says so
        plain = false;
    }
    if (!plain) return general(name, args, n);
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = fn(std::get<I>(v)...);
    Py_END_ALLOW_THREADS
    if (code == SKIPARSE_OK) Py_RETURN_NONE;
    return PyObject_CallFunction(g_failed, "is", code, name);
}

template <unsigned NONE, typename... A>
PyObject* call(int (*fn)(A...), const char* name, PyObject* const* args, Py_ssize_t n) {
    return call_with<NONE>(fn, name, args, n, std::index_sequence_for<A...>{});
}

constexpr unsigned NEVER = 0u;
constexpr unsigned at() { return 0u; }
template <typename... I>
constexpr unsigned at(int i, I... more) { return 1u << i | at(more...); }
// address of the C function: none until the binding has opened the library, and the general way is taken (which opens it)
#define SLOT(name, none) decltype(&::name) g_##name = nullptr;
// `none`: arguments that may be None, as the workspace of the forward layer, which the fused form does not need
#define ENTRY(name, none)                                                 \
    PyObject* py_##name(PyObject*, PyObject* const* args, Py_ssize_t n) { \
        return g_##name ? call<none>(g_##name, #name, args, n) : general(#name, args, n); \
    }
#define BIND(name, none) \
    if (strcmp(what, #name) == 0) g_##name = (decltype(g_##name))address;
#define LISTED(name, none) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, nullptr},
#define ENTRIES(X) \
    X(skiparse_attn_fwd, at(15)) \
    X(skiparse_permute, NEVER) \
    X(skiparse_unpermute, NEVER) \
    X(skiparse_switch_pattern, NEVER) \
    X(skiparse_ssp_pack, NEVER) \
    X(skiparse_ssp_unpack, NEVER) \
    X(dense_attn_fwd, NEVER) \
    X(skiparse_attn_fwd_sparse, NEVER) \
    X(skiparse_attn_fwd_lse, NEVER) \
    X(skiparse_attn_bwd, NEVER) \
    X(skiparse_attn_bwd_static, NEVER) \
    X(skiparse_quantize_fp8_ex, NEVER) \
    X(skiparse_attn_fwd_fp8_ex, NEVER) \
    X(skiparse_rope_table_ex, NEVER) \
    X(skiparse_rope, at(1, 3)) \
    X(skiparse_checkpoint_save, NEVER) \
    X(skiparse_checkpoint_load, NEVER) \
    X(skiparse_linear_fwd, at(2, 3, 5, 6, 18)) \
    X(skiparse_linear_bwd, at(1, 2, 3, 4, 5, 6, 7, 8, 9, 21)) \
    X(skiparse_rmsnorm_fwd, at(1, 2, 3, 5)) \
    X(skiparse_rmsnorm_bwd, at(2, 3, 4, 5, 16)) \
    X(skiparse_quantize_int8, NEVER) \
    X(skiparse_linear_fwd_int8, at(4, 5, 17))
ENTRIES(SLOT)
ENTRIES(ENTRY)

// ---- whole calls
//
// A norm of one row, its codes or its projection is a kernel of 2 to 7 us behind 8 of host work, of which the launch takes 3.5 and the results' tensors 2.5 from Python.  So these calls are here once more as a
// whole: their checks, their results' tensors and the C function.  (us a call on the host, by way of Python / so: norm with residual 7.7 / 5.2, rows in codes 8.1 / 5.4, a token's projection 8.0 / 4.4.)  plain_x(...) answers NotImplemented to anything but plain arguments that fit each other, and the binding goes on as if it had not asked: what
// is refused, and with which words, is decided there.  PLACE: None where rows stay, else (leading dimensions of the result, B, T, H, W, s, pattern, order).

decltype(&::skiparse_linear_fwd_int8_workspace_bytes) g_linear8_bytes = nullptr;
decltype(&::skiparse_rmsnorm_bwd_workspace_bytes) g_norm_bwd_bytes = nullptr;

struct Place {
    int64_t lead[2] = {0, 0};
    int B = 1, T = 1, H = 1, W = 0, s = 1, pattern = 0, order = 0;
    bool moved = false;
    bool get(PyObject* o, int64_t rows) {
        if (o == Py_None) {
            W = (int)rows;
            return rows >= 1 && W == rows;
        }
        int l[2];
        moved = true;
        if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 9) return false;
        int* const to[9] = {&l[0], &l[1], &B, &T, &H, &W, &s, &pattern, &order};
        for (int i = 0; i < 9; i++)
            if (!Arg<int>::get(PyTuple_GET_ITEM(o, i), *to[i])) return false;
        lead[0] = l[0];
        lead[1] = l[1];
        return true;
    }
    // of a result with `cols` channels, made of rows as those of `x`
    at::DimVector shape(const at::Tensor& x, int64_t cols, bool scales = false) const {
        at::DimVector d;
        if (moved) d.append(lead, lead + 2);
        else d.append(x.sizes().begin(), x.sizes().end() - 1);
        if (!scales) d.push_back(cols);
        return d;
    }
};

// Without the interpreter's lock: for the C function, and for results' tensors, whose memory can take a wait for the GPU.  It is taken again whichever way that ends, an exception from within among them.
// In a process that ends, a daemon thread that asks for it is taken off its stack instead: let through here and by PLAIN, since both would end the process in an abort otherwise.
struct Unlocked {
    PyThreadState* const state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    ~Unlocked() noexcept(false) { PyEval_RestoreThread(state); }
};

struct Here {
    int device;
    void* stream;
    // the current device, which is a number, and its stream's handle
    bool get(PyObject* get_device, PyObject* raw_stream) {
        if (get_device == Py_None || raw_stream == Py_None) return false;
        PyObject* d = PyObject_CallNoArgs(get_device);
        PyObject* h = d != nullptr ? PyObject_CallOneArg(raw_stream, d) : nullptr;
        const bool ok = h != nullptr && PyLong_CheckExact(d) && PyLong_CheckExact(h);
        if (ok) {
            device = (int)PyLong_AsLong(d);
            stream = (void*)(uintptr_t)PyLong_AsUnsignedLongLongMask(h);
        }
        Py_XDECREF(d);
        Py_XDECREF(h);
        PyErr_Clear();
        return ok;
    }
};

const at::Tensor* tensor_of(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.is_contiguous() ? &t : nullptr;
}
// like `x` in type and device; null for None
bool also(PyObject* o, const at::Tensor& x, const at::Tensor*& t, at::ScalarType type) {
    t = nullptr;
    if (o == Py_None) return true;
    t = tensor_of(o);
    return t != nullptr && t->scalar_type() == type && t->get_device() == x.get_device();
}
bool of_channels(const at::Tensor* t, int64_t cols) { return t == nullptr || (t->dim() == 1 && t->size(0) == cols); }
// Throws for a tensor without memory of its own (one inside vmap or grad, which looks like any other).
void* pointer(const at::Tensor* t) { return t != nullptr ? t->data_ptr() : nullptr; }
void* pointer(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
int elements(const at::Tensor& t) { return t.scalar_type() == at::kBFloat16 ? SKIPARSE_BF16 : t.scalar_type() == at::kFloat ? SKIPARSE_FP32 : -1; }
// (codes, scales) as the binding's class of these
PyObject* quantized(PyObject* type, at::Tensor&& codes, at::Tensor&& scales) {
    PyObject* two = PyTuple_New(2);
    if (two == nullptr) return nullptr;
    PyTuple_SET_ITEM(two, 0, THPVariable_Wrap(std::move(codes)));
    PyTuple_SET_ITEM(two, 1, THPVariable_Wrap(std::move(scales)));
    PyObject* args = PyTuple_Pack(1, two);
    PyObject* q = args != nullptr ? PyTuple_Type.tp_new((PyTypeObject*)type, args, nullptr) : nullptr;
    Py_XDECREF(args);
    Py_DECREF(two);
    return q;
}
bool quantized_of(PyObject* o, PyObject* type, const at::Tensor*& codes, const at::Tensor*& scales) {
    if ((PyObject*)Py_TYPE(o) != type || PyTuple_GET_SIZE(o) != 2) return false;
    codes = tensor_of(PyTuple_GET_ITEM(o, 0));
    scales = tensor_of(PyTuple_GET_ITEM(o, 1));
    return codes != nullptr && scales != nullptr && codes->scalar_type() == at::kChar && scales->scalar_type() == at::kFloat && codes->dim() >= 1 &&
           scales->sizes() == codes->sizes().slice(0, codes->dim() - 1) && codes->get_device() == scales->get_device();
}
bool is_class(PyObject* type) { return PyType_Check(type) && PyType_IsSubtype((PyTypeObject*)type, &PyTuple_Type); }
bool yes_or_no(PyObject* o, bool& v) {
    v = o == Py_True;
    return v || o == Py_False;
}
PyObject* not_plain() {
    Py_INCREF(Py_NotImplemented);
    return Py_NotImplemented;
}
PyObject* raised(int code, const char* name) { return PyObject_CallFunction(g_failed, "is", code, name); }

// x, weight, residual, eps, quantize, Quantized, PLACE, device and stream functions -> result, or (result, sum)
PyObject* rmsnorm_fwd_of(PyObject* const* a) {
    const at::Tensor *x = tensor_of(a[0]), *w, *r;
    bool quantize;
    if (x == nullptr || x->dim() < 1 || x->numel() < 1 || !PyFloat_CheckExact(a[3]) || !yes_or_no(a[4], quantize) || !is_class(a[5])) return not_plain();
    const int type = elements(*x);
    const int64_t cols = x->size(-1);
    Place place;
    Here here;
    if (type < 0 || cols != (int)cols || !also(a[1], *x, w, x->scalar_type()) || !of_channels(w, cols) || !also(a[2], *x, r, x->scalar_type()) || (r != nullptr && r->sizes() != x->sizes()) ||
        !place.get(a[6], x->numel() / cols) || !here.get(a[7], a[8]) || here.device != x->get_device())
        return not_plain();
    const float eps = (float)PyFloat_AS_DOUBLE(a[3]);
    at::Tensor out, scales, sum;
    int code;
    {
        const Unlocked unlocked;
        out = at::empty(place.shape(*x, cols), quantize ? x->options().dtype(at::kChar) : x->options());
        if (quantize) scales = at::empty(place.shape(*x, cols, true), x->options().dtype(at::kFloat));
        if (r != nullptr) sum = at::empty(x->sizes(), x->options());
        code = g_skiparse_rmsnorm_fwd(pointer(x), pointer(r), pointer(w), pointer(sum), pointer(out), (float*)pointer(scales), place.B, place.T, place.H, place.W, (int)cols, eps, place.s, place.pattern,
                                      place.order, type, here.stream);
    }
    if (code != SKIPARSE_OK) return raised(code, "skiparse_rmsnorm_fwd");
    PyObject* result = quantize ? quantized(a[5], std::move(out), std::move(scales)) : THPVariable_Wrap(std::move(out));
    if (result == nullptr || r == nullptr) return result;
    PyObject* both = PyTuple_New(2);
    if (both == nullptr) return nullptr;
    PyTuple_SET_ITEM(both, 0, result);
    PyTuple_SET_ITEM(both, 1, THPVariable_Wrap(std::move(sum)));
    return both;
}

// x, Quantized, PLACE, device and stream functions
PyObject* quantize_int8_of(PyObject* const* a) {
    const at::Tensor* x = tensor_of(a[0]);
    if (x == nullptr || x->dim() < 1 || x->numel() < 1 || !is_class(a[1])) return not_plain();
    const int type = elements(*x);
    const int64_t cols = x->size(-1);
    Place place;
    Here here;
    if (type < 0 || cols != (int)cols || !place.get(a[2], x->numel() / cols) || !here.get(a[3], a[4]) || here.device != x->get_device()) return not_plain();
    at::Tensor codes, scales;
    int code;
    {
        const Unlocked unlocked;
        codes = at::empty(place.shape(*x, cols), x->options().dtype(at::kChar));
        scales = at::empty(place.shape(*x, cols, true), x->options().dtype(at::kFloat));
        code = g_skiparse_quantize_int8(pointer(x), pointer(codes), (float*)pointer(scales), place.B, place.T, place.H, place.W, (int)cols, place.s, place.pattern, place.order, type, here.stream);
    }
    return code != SKIPARSE_OK ? raised(code, "skiparse_quantize_int8") : quantized(a[1], std::move(codes), std::move(scales));
}

// x, w, bias, residual, activation, Quantized, PLACE, device and stream functions.  Scales that begin off 16 bytes are the binding's to copy.
PyObject* linear_fwd_int8_of(PyObject* const* a) {
    const at::Tensor *x, *xs, *w, *ws, *bias, *residual;
    int act;
    if (!quantized_of(a[0], a[5], x, xs) || !quantized_of(a[1], a[5], w, ws) || x->numel() < 1 || w->dim() != 2 || w->get_device() != x->get_device() || !Arg<int>::get(a[4], act)) return not_plain();
    const int64_t K = x->size(-1), N = w->size(0);
    Place place;
    Here here;
    if (w->size(1) != K || K != (int)K || N != (int)N || N < 1 || !also(a[2], *x, bias, at::kBFloat16) || !of_channels(bias, N) || !also(a[3], *x, residual, at::kBFloat16) ||
        !place.get(a[6], x->numel() / K) || x->numel() / K > INT_MAX || !here.get(a[7], a[8]) || here.device != x->get_device())
        return not_plain();
    const at::DimVector shape = place.shape(*x, N);
    if (residual != nullptr && residual->sizes() != at::IntArrayRef(shape)) return not_plain();
    if ((((uintptr_t)pointer(xs) | (uintptr_t)pointer(ws)) & 15u) != 0) return not_plain();
    const size_t need = g_linear8_bytes((int)(x->numel() / K), (int)K, (int)N);
    at::Tensor space, out;
    int code;
    {
        const Unlocked unlocked;
        out = at::empty(shape, x->options().dtype(at::kBFloat16));
        if (need) space = at::empty({(int64_t)need}, x->options().dtype(at::kByte));
        code = g_skiparse_linear_fwd_int8(pointer(x), (const float*)pointer(xs), pointer(w), (const float*)pointer(ws), pointer(bias), pointer(residual), pointer(out), place.B, place.T, place.H, place.W, (int)K,
                                          (int)N, place.s, place.pattern, place.order, act, pointer(space), need, here.stream);
    }
    return code != SKIPARSE_OK ? raised(code, "skiparse_linear_fwd_int8") : THPVariable_Wrap(std::move(out));
}

// dy, h, weight, dx_add, eps, need_dx, need_dw, device and stream functions; rows stay -> (dx, dw)
PyObject* rmsnorm_bwd_of(PyObject* const* a) {
    const at::Tensor *dy = tensor_of(a[0]), *h, *w, *add;
    bool need_dx, need_dw;
    if (dy == nullptr || dy->dim() < 1 || dy->numel() < 1 || !PyFloat_CheckExact(a[4]) || !yes_or_no(a[5], need_dx) || !yes_or_no(a[6], need_dw)) return not_plain();
    const int type = elements(*dy);
    const int64_t cols = dy->size(-1);
    Place place;
    Here here;
    if (type < 0 || cols != (int)cols || !also(a[1], *dy, h, dy->scalar_type()) || h == nullptr || h->sizes() != dy->sizes() || !also(a[2], *dy, w, dy->scalar_type()) || !of_channels(w, cols) ||
        !also(a[3], *dy, add, dy->scalar_type()) || (add != nullptr && add->sizes() != dy->sizes()) || !place.get(Py_None, dy->numel() / cols) || !here.get(a[7], a[8]) || here.device != dy->get_device())
        return not_plain();
    const size_t need = need_dw ? g_norm_bwd_bytes(place.W, (int)cols) : 0;
    const float eps = (float)PyFloat_AS_DOUBLE(a[4]);
    at::Tensor dx, dw, space;
    int code;
    {
        const Unlocked unlocked;
        if (need_dx) dx = at::empty(h->sizes(), h->options());
        if (need_dw) dw = at::empty({cols}, h->options());
        if (need) space = at::empty({(int64_t)need}, h->options().dtype(at::kByte));
        code = g_skiparse_rmsnorm_bwd(pointer(dy), pointer(h), pointer(w), pointer(add), pointer(dx), pointer(dw), 1, 1, 1, place.W, (int)cols, eps, 1, 0, 0, type, pointer(space), need, here.stream);
    }
    if (code != SKIPARSE_OK) return raised(code, "skiparse_rmsnorm_bwd");
    PyObject* both = PyTuple_New(2);
    if (both == nullptr) return nullptr;
    for (int i = 0; i < 2; i++) {
        if (i ? need_dw : need_dx) {
            PyTuple_SET_ITEM(both, i, THPVariable_Wrap(i ? std::move(dw) : std::move(dx)));
        } else {
            Py_INCREF(Py_None);
            PyTuple_SET_ITEM(both, i, Py_None);
        }
    }
    return both;
}

// An exception from within (no memory for a result, a tensor without memory): the binding comes upon it by itself.
#define PLAIN(name, count, bound)                                                \
    PyObject* plain_##name(PyObject*, PyObject* const* args, Py_ssize_t n) {     \
        if (n != count || !(bound) || g_failed == nullptr) return not_plain();   \
        try {                                                                    \
            return name##_of(args);                                              \
        } catch (const abi::__forced_unwind&) { /* of a thread that is ended */  \
            throw;                                                               \
        } catch (...) {                                                          \
            PyErr_Clear();                                                       \
            return not_plain();                                                  \
        }                                                                        \
    }
PLAIN(rmsnorm_fwd, 9, g_skiparse_rmsnorm_fwd)
PLAIN(quantize_int8, 5, g_skiparse_quantize_int8)
PLAIN(linear_fwd_int8, 9, g_skiparse_linear_fwd_int8 && g_linear8_bytes)
PLAIN(rmsnorm_bwd, 9, g_skiparse_rmsnorm_bwd && g_norm_bwd_bytes)

PyObject* set_up(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 2 || !PyCallable_Check(args[0]) || !PyCallable_Check(args[1])) {
        PyErr_SetString(PyExc_TypeError, "set_up(general, failed)");
        return nullptr;
    }
    Py_INCREF(args[0]);
    Py_INCREF(args[1]);
    Py_XDECREF(g_general);
    Py_XDECREF(g_failed);
    g_general = args[0];
    g_failed = args[1];
    Py_RETURN_NONE;
}

PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    const char* what = n == 2 ? PyUnicode_AsUTF8(args[0]) : nullptr;
    void* address = what != nullptr ? PyLong_AsVoidPtr(args[1]) : nullptr;
    if (PyErr_Occurred()) return nullptr;
    if (address == nullptr) {
        PyErr_SetString(PyExc_TypeError, "bind(name, address)");
        return nullptr;
    }
    ENTRIES(BIND)
    if (strcmp(what, "skiparse_linear_fwd_int8_workspace_bytes") == 0) g_linear8_bytes = (decltype(g_linear8_bytes))address;
    if (strcmp(what, "skiparse_rmsnorm_bwd_workspace_bytes") == 0) g_norm_bwd_bytes = (decltype(g_norm_bwd_bytes))address;
    Py_RETURN_NONE;
}

#define LISTED_PLAIN(name) {"plain_" #name, (PyCFunction)(void (*)(void))plain_##name, METH_FASTCALL, nullptr},
PyMethodDef methods[] = {ENTRIES(LISTED) LISTED_PLAIN(rmsnorm_fwd) LISTED_PLAIN(quantize_int8) LISTED_PLAIN(linear_fwd_int8) LISTED_PLAIN(rmsnorm_bwd){"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
                         {"set_up", (PyCFunction)(void (*)(void))set_up, METH_FASTCALL, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Native marshalling of the binding's calls.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__marshal() {
    PyObject* m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "BUILT_FOR", BUILT_FOR) != 0) Py_CLEAR(m);
    return m;
}

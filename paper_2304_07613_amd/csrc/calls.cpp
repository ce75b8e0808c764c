// calls.cpp -- the Python side of the attention operators' C ABI: checks of
// tensors, outputs and workspace from torch's allocator, torch's current stream.
// They are called for every layer and token, where the time of a call is the
// host's: as a module the marshalling takes about 1 us, through ctypes 5 to 7.
//
// Nothing is computed here, and there is no fallback: nmg.py binds the library's
// functions (bind) when it loads it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "nmg.h"

namespace {

// The library's functions, bound when it is loaded
struct Library {
    decltype(&::nmg_rotary) rotary;
    decltype(&::nmg_qk_norm_rotary) qk_norm_rotary;
    decltype(&::nmg_attention) attention;
    decltype(&::nmg_tree_attention) tree_attention;
    decltype(&::nmg_attention_workspace_bytes) attention_workspace_bytes;
} library;
PyObject *check;          // nmg._check(status, what): raises NmgError
PyObject *current_device, *current_stream;  // torch._C's

// A refusal: the Python error is set
struct Refused {};
[[noreturn]] void refuse(PyObject *type, const char *what) {
    PyErr_SetString(type, what);
    throw Refused{};
}
[[noreturn]] void refuse_value(const char *what) { refuse(PyExc_ValueError, what); }

const at::Tensor &tensor(PyObject *o, const char *what) {
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, what);
    return THPVariable_Unpack(o);
}
const at::Tensor *maybe(PyObject *o, const char *what) {
    return o == Py_None ? nullptr : &tensor(o, what);
}
int32_t int32(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    if (v < INT32_MIN || v > INT32_MAX) refuse_value("a count does not fit 32 bits");
    return (int32_t)v;
}
double real(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{};
    return v;
}
void arguments(Py_ssize_t got, Py_ssize_t want) {
    if (got != want) refuse(PyExc_TypeError, "wrong number of arguments");
}

bool dtype_ok(const at::Tensor &t) {
    return t.scalar_type() == at::kFloat || t.scalar_type() == at::kHalf;
}
nmg_dtype dtype_of(const at::Tensor &t) { return t.scalar_type() == at::kFloat ? NMG_F32 : NMG_F16; }
const char *const kMatrix = "a matrix must be a 2-D tensor with unit column stride";

// Leading dimension of a 2-D row-major tensor
int64_t rows(const at::Tensor &t, const char *what) {
    if (t.dim() != 2 || t.stride(1) != 1) refuse_value(what);
    return t.stride(0);
}
const int32_t *ints(const at::Tensor &t, int64_t n, const char *what) {
    if (t.scalar_type() != at::kInt || t.dim() != 1 || t.numel() != n || !t.is_contiguous())
        refuse_value(what);
    return t.data_ptr<int32_t>();
}
int64_t head_rows(int64_t all, int64_t heads) {
    if (heads < 1 || all < 1 || all % heads)
        refuse_value("a matrix must have a whole number of rows for each of its heads");
    return all / heads;
}

// Every tensor of a call on the current GPU; its current stream
struct Gpu {
    int device = -2;
    void operator()(const at::Tensor &t) {
        if (!t.is_cuda()) refuse_value("libnmg works on GPU tensors only");
        const int d = t.get_device();
        if (device == -2) {
            PyObject *now = PyObject_CallNoArgs(current_device);
            if (!now) throw Refused{};
            const long v = PyLong_AsLong(now);
            Py_DECREF(now);
            if (v == -1 && PyErr_Occurred()) throw Refused{};
            device = (int)v;
        }
        if (d != device)
            refuse_value("a tensor is not on the current device (select it with torch.cuda.device)");
    }
    hipStream_t stream() const {
        PyObject *index = PyLong_FromLong(device);
        if (!index) throw Refused{};
        PyObject *raw = PyObject_CallOneArg(current_stream, index);
        Py_DECREF(index);
        if (!raw) throw Refused{};
        void *s = PyLong_AsVoidPtr(raw);
        Py_DECREF(raw);
        if (!s && PyErr_Occurred()) throw Refused{};
        return (hipStream_t)s;
    }
};

// Without the interpreter lock: memory is allocated and kernels are launched then, and
// nothing of Python's is touched.  (A launch may wait, and so may the allocator.)
struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked &) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// The output that was given, checked; undefined if none was
at::Tensor output(Gpu &gpu, const at::Tensor &like, const at::Tensor *given) {
    if (!given) return at::Tensor();
    if (given->scalar_type() != like.scalar_type() || given->sizes() != like.sizes())
        refuse_value("an output must have the shape and dtype of its input");
    gpu(*given);
    (void)rows(*given, kMatrix);
    return *given;
}
// (called Unlocked)
void allocate(at::Tensor &y, const at::Tensor &like) {
    if (!y.defined()) y = at::empty_like(like, at::MemoryFormat::Contiguous);
}

void checked(nmg_status status, const char *what) {
    if (status == NMG_OK) return;
    PyObject *r = PyObject_CallFunction(check, "is", (int)status, what);
    Py_XDECREF(r);
    if (r) PyErr_SetString(PyExc_RuntimeError, what);
    throw Refused{};
}

nmg_rotary_desc rotary_desc(Gpu &gpu, PyObject *table, PyObject *positions, PyObject *pairs, int64_t N) {
    nmg_rotary_desc r = {0, NMG_ROTARY_HALF, 0, nullptr, nullptr};
    if (!PyUnicode_Check(pairs)) refuse_value("unknown rotary layout");
    if (PyUnicode_CompareWithASCIIString(pairs, "interleaved") == 0)
        r.pairs = NMG_ROTARY_INTERLEAVED;
    else if (PyUnicode_CompareWithASCIIString(pairs, "half") != 0)
        refuse_value("unknown rotary layout");
    const at::Tensor *t = maybe(table, "table must be a tensor or None");
    if (!t) return r;
    if (t->dim() != 3 || t->size(0) != 2 || t->scalar_type() != at::kFloat || !t->is_contiguous())
        refuse_value("table must be a contiguous float32 (2, dim / 2, length) tensor");
    const at::Tensor &p = tensor(positions, "positions must be a tensor");
    r.dim = (int32_t)(2 * t->size(1));
    r.length = t->size(2);
    r.table = t->data_ptr<float>();
    r.positions = ints(p, N, "positions must be N contiguous int32 values");
    gpu(*t);
    gpu(p);
    return r;
}

at::Tensor rotary(PyObject *const *a) {
    const at::Tensor &x = tensor(a[0], "X must be a tensor");
    if (!dtype_ok(x)) refuse(PyExc_TypeError, "X must be float32 or float16");
    const int64_t ldx = rows(x, kMatrix), N = x.size(1);
    const int32_t heads = int32(a[1]);
    const int64_t D = head_rows(x.size(0), heads);
    Gpu gpu;
    const nmg_rotary_desc r = rotary_desc(gpu, a[2], a[3], a[4], N);
    gpu(x);
    at::Tensor y = output(gpu, x, maybe(a[5], "out must be a tensor"));
    const hipStream_t stream = gpu.stream();
    nmg_status status;
    {
        Unlocked now;
        allocate(y, x);
        status = library.rotary(dtype_of(x), heads, (int32_t)D, &r, x.data_ptr(), ldx, N, y.data_ptr(),
                            y.stride(0), stream);
    }
    checked(status, "nmg_rotary");
    return y;
}

std::pair<at::Tensor, at::Tensor> qk_norm_rotary(PyObject *const *a) {
    const at::Tensor &q = tensor(a[0], "Q must be a tensor"), &k = tensor(a[1], "K must be a tensor");
    if (!dtype_ok(q) || k.scalar_type() != q.scalar_type())
        refuse(PyExc_TypeError, "Q and K must be float32 or float16, of one dtype");
    const int64_t ldq = rows(q, kMatrix), ldk = rows(k, kMatrix), N = q.size(1);
    const int32_t heads = int32(a[2]), kv_heads = int32(a[3]);
    const int64_t D = head_rows(q.size(0), heads);
    if (k.size(1) != N || head_rows(k.size(0), kv_heads) != D)
        refuse_value("Q and K must have heads of one size and the same tokens");
    Gpu gpu;
    const float *weights[2];
    for (int i = 0; i < 2; ++i) {
        const at::Tensor *w = maybe(a[4 + i], "norm weights must be tensors or None");
        weights[i] = nullptr;
        if (!w) continue;
        if (w->scalar_type() != at::kFloat || w->dim() != 1 || w->numel() != D || !w->is_contiguous())
            refuse_value("norm weights must be head_dim contiguous float32 values");
        gpu(*w);
        weights[i] = w->data_ptr<float>();
    }
    const nmg_rotary_desc r = rotary_desc(gpu, a[6], a[7], a[8], N);
    const double eps = real(a[9]);
    gpu(q);
    gpu(k);
    at::Tensor yq = output(gpu, q, maybe(a[10], "out[0] must be a tensor"));
    at::Tensor yk = output(gpu, k, maybe(a[11], "out[1] must be a tensor"));
    const hipStream_t stream = gpu.stream();
    nmg_status status;
    {
        Unlocked now;
        allocate(yq, q);
        allocate(yk, k);
        status = library.qk_norm_rotary(dtype_of(q), heads, kv_heads, (int32_t)D, &r, weights[0], weights[1],
                                    (float)eps, q.data_ptr(), ldq, k.data_ptr(), ldk, N,
                                    yq.data_ptr(), yq.stride(0), yk.data_ptr(), yk.stride(0), stream);
    }
    checked(status, "nmg_qk_norm_rotary");
    return {yq, yk};
}

bool bytes(const at::Tensor &t) {
    return t.scalar_type() == at::kByte || t.scalar_type() == at::kBool;
}

at::Tensor attention(PyObject *const *a) {
    const at::Tensor &q = tensor(a[0], "Q must be a tensor"), &k = tensor(a[1], "K must be a tensor"),
                     &v = tensor(a[2], "V must be a tensor");
    nmg_heads h = {int32(a[3]), int32(a[4]), 0, dtype_of(q)};
    if (!dtype_ok(q) || k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type())
        refuse(PyExc_TypeError, "Q, K and V must be float32 or float16, of one dtype");
    const int64_t ldq = rows(q, kMatrix), ldk = rows(k, kMatrix), ldv = rows(v, kMatrix);
    const int64_t Nq = q.size(1), Nk = k.size(1), D = head_rows(q.size(0), h.heads);
    if (v.sizes() != k.sizes() || head_rows(k.size(0), h.kv_heads) != D)
        refuse_value("K and V must have kv_heads heads of Q's head size, and the same tokens");
    h.head_dim = (int32_t)std::min<int64_t>(D, INT32_MAX);
    const at::Tensor &offsets = tensor(a[5], "q_offsets must be a tensor"),
                     &begin = tensor(a[6], "kv_begin must be a tensor"),
                     &end = tensor(a[7], "kv_end must be a tensor");
    const int64_t B = begin.numel();
    if (B > INT32_MAX) refuse_value("too many sequences");
    const nmg_sequences s = {(int32_t)B,
                         ints(offsets, B + 1, "q_offsets must be one more contiguous int32 value than kv_begin has"),
                         ints(begin, B, "kv_begin must be contiguous int32 values"),
                         ints(end, B, "kv_end must be as many contiguous int32 values as kv_begin")};
    Gpu gpu;
    gpu(q);
    gpu(k);
    gpu(v);
    gpu(offsets);
    gpu(begin);
    gpu(end);
    const at::Tensor *mask = maybe(a[8], "key_mask must be a tensor or None");
    const at::Tensor *tree = maybe(a[9], "tree must be a tensor");
    if (mask) {
        if (!bytes(*mask) || mask->dim() != 1 || mask->numel() != Nk || !mask->is_contiguous())
            refuse_value("key_mask must be contiguous uint8 or bool, one for every key column");
        gpu(*mask);
    }
    int64_t ldtree = 0;
    if (tree) {
        if (!bytes(*tree) || tree->dim() != 2 || tree->size(0) != Nq)
            refuse_value("tree must be uint8 or bool with a row for every query column");
        ldtree = rows(*tree, kMatrix);
        gpu(*tree);
    }
    const float scale = a[10] == Py_None ? (float)(1.0 / std::sqrt((double)D)) : (float)real(a[10]);
    at::Tensor o = output(gpu, q, maybe(a[11], "out must be a tensor"));
    const hipStream_t stream = gpu.stream();
    nmg_status status;
    {
        Unlocked now;
        allocate(o, q);
        // freed after the call returns: the allocator hands it out again in stream order
        at::Tensor space;
        int64_t room = library.attention_workspace_bytes(&h, s.count, Nq, Nk);
        if (room > 0) {
            try {
                space = at::empty({room}, q.options().dtype(at::kByte));
            } catch (const c10::OutOfMemoryError &) {
                room = 0;
            }
        }
        void *ws = room > 0 ? space.data_ptr() : nullptr;
        room = std::max<int64_t>(room, 0);
        if (tree)
            status = library.tree_attention(&h, &s, q.data_ptr(), ldq, Nq, k.data_ptr(), ldk, v.data_ptr(),
                                        ldv, Nk, (const uint8_t *)tree->data_ptr(), ldtree, tree->size(1), scale,
                                        o.data_ptr(), o.stride(0), ws, room, stream);
        else
            status = library.attention(&h, &s, q.data_ptr(), ldq, Nq, k.data_ptr(), ldk, v.data_ptr(), ldv,
                                   Nk, mask ? (const uint8_t *)mask->data_ptr() : nullptr, scale, o.data_ptr(),
                                   o.stride(0), ws, room, stream);
    }
    checked(status, tree ? "nmg_tree_attention" : "nmg_attention");
    return o;
}

// No C++ exception leaves a call
template <typename F>
PyObject *guarded(F f) {
    try {
        at::AutoDispatchBelowADInplaceOrView plain;  // no autograd: outputs have no gradient
        return f();
    } catch (const Refused &) {
        return nullptr;
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(PyExc_MemoryError, e.what());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

PyObject *py_rotary(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        arguments(n, 6);
        return THPVariable_Wrap(rotary(a));
    });
}
PyObject *py_qk_norm_rotary(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        arguments(n, 12);
        auto y = qk_norm_rotary(a);
        PyObject *q = THPVariable_Wrap(y.first), *k = q ? THPVariable_Wrap(y.second) : nullptr;
        PyObject *both = k ? PyTuple_Pack(2, q, k) : nullptr;
        Py_XDECREF(q);
        Py_XDECREF(k);
        return both;
    });
}
PyObject *py_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&] {
        arguments(n, 12);
        return THPVariable_Wrap(attention(a));
    });
}

// bind(functions, check, current_device, current_stream): addresses of the
// library's functions by name, nmg._check, and torch._C's two
PyObject *py_bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        arguments(n, 4);
        auto at = [&](const char *name) {
            PyObject *v = PyDict_Check(a[0]) ? PyDict_GetItemString(a[0], name) : nullptr;
            void *p = v ? PyLong_AsVoidPtr(v) : nullptr;
            if (!p) refuse_value(name);
            return p;
        };
        auto bound = [&](auto &f, const char *name) { f = (std::decay_t<decltype(f)>)at(name); };
        bound(library.rotary, "nmg_rotary");
        bound(library.qk_norm_rotary, "nmg_qk_norm_rotary");
        bound(library.attention, "nmg_attention");
        bound(library.tree_attention, "nmg_tree_attention");
        bound(library.attention_workspace_bytes, "nmg_attention_workspace_bytes");
        PyObject **kept[3] = {&check, &current_device, &current_stream};
        for (int i = 0; i < 3; ++i) {
            Py_INCREF(a[1 + i]);
            Py_XDECREF(*kept[i]);
            *kept[i] = a[1 + i];
        }
        Py_RETURN_NONE;
    });
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)())py_bind, METH_FASTCALL, nullptr},
    {"rotary", (PyCFunction)(void (*)())py_rotary, METH_FASTCALL, nullptr},
    {"qk_norm_rotary", (PyCFunction)(void (*)())py_qk_norm_rotary, METH_FASTCALL, nullptr},
    {"attention", (PyCFunction)(void (*)())py_attention, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr,
                      nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) { return PyModule_Create(&module); }

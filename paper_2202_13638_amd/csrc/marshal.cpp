// Checks of tensor arguments and their packing into the C ABI's structures (include/bagel.h), for binding.py: what takes half a microsecond a
// tensor in Python takes some ten nanoseconds here, and calls of a few rows, or updates of a hundred small tensors, consist of little else.
// Errors are Python's ValueError; nothing here touches the GPU.
#include <Python.h>

#include <algorithm>
#include <cstdint>
#include <cstring>
#include <string>
#include <vector>

#include <torch/csrc/autograd/python_variable.h>

#include "bagel.h"

namespace {

std::string shown(const at::IntArrayRef &sizes)
{
    std::string s = "(";
    for (size_t i = 0; i < sizes.size(); ++i) s += (i ? ", " : "") + std::to_string(sizes[i]);
    return s + (sizes.size() == 1 ? ",)" : ")");
}

std::string type_name(at::ScalarType t)
{
    switch (t) {
    case at::kFloat: return "float32";
    case at::kBFloat16: return "bfloat16";
    case at::kHalf: return "float16";
    case at::kFloat8_e4m3fn: return "float8_e4m3fn";
    default: return c10::toString(t);
    }
}

struct refused {
    std::string message;
};

const at::Tensor &tensor_of(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) throw refused{std::string(name) + " must be a tensor"};
    return THPVariable_Unpack(o);
}

bool on(const at::Tensor &t, int64_t device) { return t.is_cuda() && t.get_device() == device; }

[[noreturn]] void refuse(const char *name, const at::Tensor &t, const std::string &wanted)
{
    throw refused{std::string(name) + " must be " + wanted + ", not " + type_name(t.scalar_type()) + " of " + shown(t.sizes()) + " on " + t.device().str()};
}

const char *name_of(PyObject *names, Py_ssize_t i) { return PyUnicode_AsUTF8(PyTuple_GET_ITEM(names, i)); }

int type_code(at::ScalarType t) { return t == at::kFloat ? BAGEL_FLOAT32 : t == at::kBFloat16 ? BAGEL_BFLOAT16 : t == at::kHalf ? BAGEL_FLOAT16 : -1; }

// Whatever goes wrong in C++ becomes an exception of Python's.
template <typename F> PyObject *guarded(F &&f)
{
    try {
        return f();
    } catch (const refused &r) {
        PyErr_SetString(PyExc_ValueError, r.message.c_str());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

PyObject *bytes_of(const std::vector<int64_t> &v) { return PyBytes_FromStringAndSize((const char *)v.data(), (Py_ssize_t)(v.size() * sizeof(int64_t))); }

// first(tensor, name, device) -> (rows, width, type code) of a matrix
PyObject *first(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 3) throw refused{"first(tensor, name, device)"};
        const char *name = PyUnicode_AsUTF8(args[1]);
        const int64_t device = PyLong_AsLongLong(args[2]);
        if (!THPVariable_Check(args[0]) || type_code(THPVariable_Unpack(args[0]).scalar_type()) < 0)
            throw refused{std::string(name) + " must be a float32, bfloat16 or float16 tensor"};
        const at::Tensor &t = THPVariable_Unpack(args[0]);
        if (!on(t, device)) throw refused{std::string(name) + " must be on the current GPU"};
        if (t.dim() != 2) throw refused{std::string(name) + " must have two dimensions, rows and width, not " + std::to_string(t.dim())};
        return Py_BuildValue("LLi", (long long)t.size(0), (long long)t.size(1), type_code(t.scalar_type()));
    });
}

// matrices(like, names, tensors) -> a bagel_matrix for each, of the shape, type and device of `like`; None: left out
PyObject *matrices(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 3 || !PyTuple_Check(args[1]) || !PyTuple_Check(args[2]) || PyTuple_GET_SIZE(args[1]) != PyTuple_GET_SIZE(args[2]))
            throw refused{"matrices(like, names, tensors)"};
        const at::Tensor &like = tensor_of(args[0], "like");
        const int64_t device = like.get_device(), rows = like.size(0), width = like.size(1);
        std::vector<int64_t> out;
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(args[2]); ++i) {
            PyObject *o = PyTuple_GET_ITEM(args[2], i);
            if (o == Py_None) {
                out.insert(out.end(), {0, 0});
                continue;
            }
            const char *name = name_of(args[1], i);
            const at::Tensor &t = tensor_of(o, name);
            if (t.scalar_type() != like.scalar_type() || t.sizes() != like.sizes() || !on(t, device))
                refuse(name, t, "a " + type_name(like.scalar_type()) + " tensor of shape " + shown(like.sizes()) + " on " + like.device().str());
            if (t.stride(1) != 1 && width > 1 && rows > 0) throw refused{std::string(name) + ": the entries of a row must be next to each other"};
            out.insert(out.end(), {(int64_t)(intptr_t)t.data_ptr(), rows > 1 ? t.stride(0) : width});
        }
        return bytes_of(out);
    });
}

// vectors(device, shape, names, tensors) -> a pointer for each, contiguous float32 of that shape; None: null
PyObject *vectors(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 4 || !PyTuple_Check(args[1]) || !PyTuple_Check(args[2]) || !PyTuple_Check(args[3]) || PyTuple_GET_SIZE(args[2]) != PyTuple_GET_SIZE(args[3]))
            throw refused{"vectors(device, shape, names, tensors)"};
        const int64_t device = PyLong_AsLongLong(args[0]);
        std::vector<int64_t> shape, out;
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(args[1]); ++i) shape.push_back(PyLong_AsLongLong(PyTuple_GET_ITEM(args[1], i)));
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(args[3]); ++i) {
            PyObject *o = PyTuple_GET_ITEM(args[3], i);
            if (o == Py_None) {
                out.push_back(0);
                continue;
            }
            const char *name = name_of(args[2], i);
            const at::Tensor &t = tensor_of(o, name);
            if (t.scalar_type() != at::kFloat || t.sizes() != at::IntArrayRef(shape) || !on(t, device) || !t.is_contiguous())
                refuse(name, t, "a contiguous float32 tensor of shape " + shown(shape) + " on cuda:" + std::to_string(device));
            out.push_back((int64_t)(intptr_t)t.data_ptr());
        }
        return bytes_of(out);
    });
}

// heads(device, type code, rows, names, (heads, width, heads, width, ...), tensors) -> a bagel_heads for each, of shape [rows, heads, width]; None: left out
PyObject *heads(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 6 || !PyTuple_Check(args[3]) || !PyTuple_Check(args[4]) || !PyTuple_Check(args[5]) || PyTuple_GET_SIZE(args[3]) != PyTuple_GET_SIZE(args[5]) ||
            PyTuple_GET_SIZE(args[4]) != 2 * PyTuple_GET_SIZE(args[5]))
            throw refused{"heads(device, type code, rows, names, sizes, tensors)"};
        const int64_t device = PyLong_AsLongLong(args[0]), code = PyLong_AsLongLong(args[1]), rows = PyLong_AsLongLong(args[2]);
        const at::ScalarType type = code == BAGEL_FLOAT32 ? at::kFloat : code == BAGEL_BFLOAT16 ? at::kBFloat16 : at::kHalf;
        std::vector<int64_t> out;
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(args[5]); ++i) {
            PyObject *o = PyTuple_GET_ITEM(args[5], i);
            if (o == Py_None) {
                out.insert(out.end(), {0, 0, 0});
                continue;
            }
            const char *name = name_of(args[3], i);
            const at::Tensor &t = tensor_of(o, name);
            const int64_t shape[3] = {rows, PyLong_AsLongLong(PyTuple_GET_ITEM(args[4], 2 * i)), PyLong_AsLongLong(PyTuple_GET_ITEM(args[4], 2 * i + 1))};
            if (t.scalar_type() != type || t.sizes() != at::IntArrayRef(shape, 3) || !on(t, device))
                refuse(name, t, "a " + type_name(type) + " tensor of shape " + shown(at::IntArrayRef(shape, 3)) + " on cuda:" + std::to_string(device));
            if (t.stride(2) != 1 && shape[2] > 1 && rows > 0) throw refused{std::string(name) + ": the entries of a head must be next to each other"};
            const int64_t head = shape[1] > 1 ? t.stride(1) : shape[2];
            out.insert(out.end(), {(int64_t)(intptr_t)t.data_ptr(), rows > 1 ? t.stride(0) : head * shape[1], head});
        }
        return bytes_of(out);
    });
}

// Whether two tensors of heads, of as many rows, have an entry in the same place.  Where their rows or heads are different distances apart it is not found out (false), unless
// one lies behind the other: parts of one projection have the same.
bool meet(const at::Tensor &x, const at::Tensor &y)
{
    struct place {
        int64_t rows, heads, width, stride, head;
        explicit place(const at::Tensor &t) : rows(t.size(0)), heads(t.size(1)), width(t.size(2)), stride(rows > 1 ? t.stride(0) : 0), head(heads > 1 ? t.stride(1) : 0) {}
        int64_t reach() const { return (rows - 1) * stride + (heads - 1) * head + width; }
    };
    if (x.numel() == 0 || y.numel() == 0) return false;
    const place a(x), b(y);
    const int64_t bytes = x.element_size(), apart = (int64_t)((intptr_t)y.data_ptr() - (intptr_t)x.data_ptr());
    if (apart >= a.reach() * bytes || -apart >= b.reach() * bytes) return false;
    if (a.stride != b.stride || (a.heads > 1 && b.heads > 1 && a.head != b.head)) return false;
    const int64_t head = a.heads > 1 ? a.head : b.head;
    for (int64_t h = 1 - b.heads; h < a.heads; ++h) {                 // the difference of their heads, and those of their rows at which such heads are nearest
        const int64_t off = h * head * bytes - apart, row = a.stride * bytes, nearest = row > 0 ? -off / row : 0;
        for (int64_t r = std::max(nearest - 1, 1 - a.rows); r <= std::min(nearest + 1, a.rows - 1); ++r) {
            const int64_t from = r * row + off;                       // from an entry of y to one of x
            if (from < b.width * bytes && -from < a.width * bytes) return true;
        }
    }
    return false;
}

// apart(names, results, names, tensors): refuses results in the place of one of the tensors, or of each other; None: left out
PyObject *apart(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 4 || !PyTuple_Check(args[0]) || !PyTuple_Check(args[1]) || !PyTuple_Check(args[2]) || !PyTuple_Check(args[3])) throw refused{"apart(names, results, names, tensors)"};
        const Py_ssize_t results = PyTuple_GET_SIZE(args[1]), others = PyTuple_GET_SIZE(args[3]);
        for (Py_ssize_t i = 0; i < results; ++i) {
            PyObject *const o = PyTuple_GET_ITEM(args[1], i);
            if (o == Py_None) continue;
            for (Py_ssize_t j = i + 1; j < results + others; ++j) {
                PyObject *const other = j < results ? PyTuple_GET_ITEM(args[1], j) : PyTuple_GET_ITEM(args[3], j - results);
                if (other == Py_None || !meet(THPVariable_Unpack(o), THPVariable_Unpack(other))) continue;
                throw refused{std::string(name_of(args[0], i)) + " may not be in the place of " + (j < results ? name_of(args[0], j) : name_of(args[2], j - results))};
            }
        }
        Py_RETURN_NONE;
    });
}

// first_heads(tensor, name, device) -> (rows, heads, width, type code) of a tensor of heads
PyObject *first_heads(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 3) throw refused{"first_heads(tensor, name, device)"};
        const char *name = PyUnicode_AsUTF8(args[1]);
        const int64_t device = PyLong_AsLongLong(args[2]);
        if (!THPVariable_Check(args[0]) || type_code(THPVariable_Unpack(args[0]).scalar_type()) < 0)
            throw refused{std::string(name) + " must be a float32, bfloat16 or float16 tensor"};
        const at::Tensor &t = THPVariable_Unpack(args[0]);
        if (!on(t, device)) throw refused{std::string(name) + " must be on the current GPU"};
        if (t.dim() != 3) throw refused{std::string(name) + " must have three dimensions, rows, heads and width, not " + std::to_string(t.dim())};
        return Py_BuildValue("LLLi", (long long)t.size(0), (long long)t.size(1), (long long)t.size(2), type_code(t.scalar_type()));
    });
}

struct list {
    PyObject *items = nullptr;               // a list or tuple, or null
    list() = default;
    list(const list &) = delete;
    ~list() { Py_XDECREF(items); }
    // None is nothing at all, where nothing is wanted; whatever else is given has to be a sequence of n entries.
    void of(PyObject *o, Py_ssize_t n, bool wanted, const char *name)
    {
        if (o != Py_None) {
            items = PySequence_Fast(o, "");
            PyErr_Clear();
        }
        if (items ? PySequence_Fast_GET_SIZE(items) != n : wanted || o != Py_None)
            throw refused{std::string("the lists of one update must have an entry for every tensor, ") + name +
                          " does not (moments in 8 bits need m_scale and v_scale)"};
    }
    // A list of one entry for every gradient, or None.
    void beside(PyObject *o, Py_ssize_t n, const char *name)
    {
        if (o == Py_None) return;
        items = PySequence_Fast(o, "");
        PyErr_Clear();
        if (!items || PySequence_Fast_GET_SIZE(items) != n) throw refused{std::string(name) + " must be a list with an entry for every gradient"};
    }
    // A list that has no place in this update: of the right length, and nothing in it.
    void none(PyObject *o, Py_ssize_t n, const char *name)
    {
        of(o, n, false, name);
        for (Py_ssize_t i = 0; items && i < n; ++i)
            if ((*this)[i] != Py_None) throw refused{std::string(name) + " belongs to moments in 8 bits"};
    }
    PyObject *operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(items, i); }
};

// adamw(device, params, grads, m, v, m_scale, v_scale, copy, weight_decay) -> (n, bagel_adamw_tensor for each, type codes of grads and copy, bits of the moments)
PyObject *adamw(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    return guarded([&]() -> PyObject * {
        if (n_args != 9) throw refused{"adamw(device, params, grads, m, v, m_scale, v_scale, copy, weight_decay)"};
        const int64_t device = PyLong_AsLongLong(args[0]);
        const Py_ssize_t n = PySequence_Size(args[1]);
        if (n < 0) return nullptr;
        list p, g, m, v, m_scale, v_scale, copy, decay;
        p.of(args[1], n, true, "params");
        g.of(args[2], n, true, "grads");
        m.of(args[3], n, true, "m");
        v.of(args[4], n, true, "v");
        const bool eight = n > 0 && tensor_of(m[0], "m").scalar_type() == at::kFloat8_e4m3fn;
        if (eight) {
            m_scale.of(args[5], n, true, "m_scale");
            v_scale.of(args[6], n, true, "v_scale");
        } else {
            m_scale.none(args[5], n, "m_scale");
            v_scale.none(args[6], n, "v_scale");
        }
        copy.of(args[7], n, false, "copy");
        const bool one_decay = PyFloat_Check(args[8]) || PyLong_Check(args[8]);
        if (!one_decay) decay.of(args[8], n, true, "weight_decay");
        const double each_decay = one_decay ? PyFloat_AsDouble(args[8]) : 0.0;
        const at::ScalarType state = eight ? at::kFloat8_e4m3fn : at::kFloat;
        at::ScalarType grad_type = at::kFloat, copy_type = at::kFloat;
        if (n > 0) {
            grad_type = tensor_of(g[0], "grads").scalar_type();
            if (type_code(grad_type) < 0) throw refused{"grads must be float32, bfloat16 or float16 tensors"};
            if (copy.items) copy_type = tensor_of(copy[0], "copy").scalar_type();
            if (type_code(copy_type) < 0) throw refused{"copy must be float32, bfloat16 or float16 tensors"};
        }
        PyObject *table = PyBytes_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(bagel_adamw_tensor));
        if (!table) return nullptr;
        try {
            bagel_adamw_tensor *to = (bagel_adamw_tensor *)PyBytes_AS_STRING(table);
            for (Py_ssize_t i = 0; i < n; ++i) {
                const at::Tensor &param = tensor_of(p[i], "params");
                const auto held = [&](PyObject *o, const char *name, at::ScalarType type) {
                    const at::Tensor &t = tensor_of(o, name);
                    if (t.scalar_type() != type || t.sizes() != param.sizes() || !t.is_contiguous() || !on(t, device))
                        refuse(("tensor " + std::to_string(i) + " of an update: " + name).c_str(), t,
                               "a contiguous " + type_name(type) + " tensor of shape " + shown(param.sizes()) + " on cuda:" + std::to_string(device));
                    return t.data_ptr();
                };
                bagel_adamw_tensor x;
                std::memset(&x, 0, sizeof(x));
                x.param = (float *)held(p[i], "params", at::kFloat);
                x.grad = held(g[i], "grads", grad_type);
                x.m = held(m[i], "m", state);
                x.v = held(v[i], "v", state);
                x.count = param.numel();
                if (eight) {
                    const int64_t blocks = (x.count + BAGEL_ADAMW_BLOCK - 1) / BAGEL_ADAMW_BLOCK;
                    const auto scales = [&](PyObject *o, const char *name) {
                        const at::Tensor &t = tensor_of(o, name);
                        if (t.scalar_type() != at::kFloat || t.numel() != blocks || !t.is_contiguous() || !on(t, device))
                            refuse(("tensor " + std::to_string(i) + " of an update: " + name).c_str(), t,
                                   "a contiguous float32 tensor of " + std::to_string(blocks) + " values on cuda:" + std::to_string(device));
                        return (float *)t.data_ptr();
                    };
                    x.m_scale = scales(m_scale[i], "m_scale");
                    x.v_scale = scales(v_scale[i], "v_scale");
                }
                if (copy.items) x.copy = held(copy[i], "copy", copy_type);
                x.weight_decay = one_decay ? each_decay : PyFloat_AsDouble(decay[i]);
                to[i] = x;
            }
        } catch (...) {
            Py_DECREF(table);
            throw;
        }
        if (PyErr_Occurred()) {              // a weight decay that is no number
            Py_DECREF(table);
            return nullptr;
        }
        return Py_BuildValue("nNiii", n, table, type_code(grad_type), type_code(copy_type), eight ? 8 : 32);
    });
}

// clip(device, grads, out) -> (n, bagel_clip_tensor for each)
PyObject *clip(PyObject *, PyObject *const *args, Py_ssize_t n_args)
{
    return guarded([&]() -> PyObject * {
        if (n_args != 3) throw refused{"clip(device, grads, out)"};
        const int64_t device = PyLong_AsLongLong(args[0]);
        const Py_ssize_t n = THPVariable_Check(args[1]) ? -1 : PySequence_Size(args[1]);
        if (n < 0) {
            PyErr_Clear();
            throw refused{"grads must be a list of tensors"};
        }
        list g, out;
        g.beside(args[1], n, "grads");
        out.beside(args[2], n, "out");
        PyObject *table = PyBytes_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(bagel_clip_tensor));
        if (!table) return nullptr;
        try {
            bagel_clip_tensor *to = (bagel_clip_tensor *)PyBytes_AS_STRING(table);
            for (Py_ssize_t i = 0; i < n; ++i) {
                const at::Tensor &grad = tensor_of(g[i], "grads");
                const at::ScalarType type = grad.scalar_type();
                if (type_code(type) < 0) throw refused{"grads must be float32, bfloat16 or float16 tensors"};
                const auto held = [&](PyObject *o, const char *name) {
                    const at::Tensor &t = tensor_of(o, name);
                    if (t.scalar_type() != type || t.sizes() != grad.sizes() || !t.is_contiguous() || !on(t, device))
                        refuse(("tensor " + std::to_string(i) + " of the gradients: " + name).c_str(), t,
                               "a contiguous " + type_name(type) + " tensor of shape " + shown(grad.sizes()) + " on cuda:" + std::to_string(device));
                    return t.data_ptr();
                };
                bagel_clip_tensor x;
                std::memset(&x, 0, sizeof(x));
                x.grad = held(g[i], "grads");
                x.out = out.items && out[i] != Py_None ? held(out[i], "out") : nullptr;
                x.count = grad.numel();
                x.dtype = type_code(type);
                to[i] = x;
            }
        } catch (...) {
            Py_DECREF(table);
            throw;
        }
        return Py_BuildValue("nN", n, table);
    });
}

PyMethodDef METHODS[] = {{"first", (PyCFunction)(void *)first, METH_FASTCALL, nullptr},
                         {"matrices", (PyCFunction)(void *)matrices, METH_FASTCALL, nullptr},
                         {"vectors", (PyCFunction)(void *)vectors, METH_FASTCALL, nullptr},
                         {"first_heads", (PyCFunction)(void *)first_heads, METH_FASTCALL, nullptr},
                         {"heads", (PyCFunction)(void *)heads, METH_FASTCALL, nullptr},
                         {"apart", (PyCFunction)(void *)apart, METH_FASTCALL, nullptr},
                         {"clip", (PyCFunction)(void *)clip, METH_FASTCALL, nullptr},
                         {"adamw", (PyCFunction)(void *)adamw, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef MODULE = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of binding.py.", -1, METHODS, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&MODULE); }

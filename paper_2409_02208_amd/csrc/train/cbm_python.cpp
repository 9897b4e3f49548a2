// CPython module of the calls between the products: reads the addresses, shapes, strides and types of PyTorch tensors, refuses what the C ABI cannot see, and calls it.  A small call's
// time is the host's: with tensors read in Python and arguments converted by ctypes, cbm_layer_norm of 1024 x 64 took
// 7.1 us a call, here it takes 3.8 to 4.1, as long as filling a tensor of one float.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <algorithm>
#include <cstdint>
#include <sstream>
#include <string>

#include "cbm.h"

namespace {

struct Refused {  // becomes a ValueError
    std::string why;
};

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) throw Refused{std::string(name) + " must be a tensor"};
    return THPVariable_Unpack(o);
}

int type_of(at::ScalarType t) { return t == at::kFloat ? CBM_F32 : t == at::kBFloat16 ? CBM_BF16 : t == at::kHalf ? CBM_F16 : -1; }
// the C ABI has rows of 32 bits, and refuses any as long as this
int32_t columns(int64_t k) { return (int32_t)std::min<int64_t>(k, INT32_MAX); }

struct Matrix {
    void* p;
    int64_t ld, rows, cols;
    int32_t type;
    bool alike(const Matrix& o) const { return rows == o.rows && cols == o.cols && type == o.type; }
};
// A device matrix of the type `only`, or of one of the three types of a cbm_dtype.
Matrix matrix(PyObject* o, const char* name, at::ScalarType only = at::ScalarType::Undefined) {
    const at::Tensor& t = tensor(o, name);
    const bool any = only == at::ScalarType::Undefined;
    const int type = any ? type_of(t.scalar_type()) : t.scalar_type() == only ? 0 : -1;
    if (type >= 0 && t.is_cuda() && t.layout() == at::kStrided && t.dim() == 2) {
        const int64_t rows = t.size(0), cols = t.size(1), ld = t.stride(0);
        if (t.stride(1) == 1 || cols <= 1) return {t.data_ptr(), rows > 1 || ld > cols ? ld : cols, rows, cols, type};
    }
    throw Refused{std::string(name) + " must be a 2-D device tensor of " + (any ? "float32, bfloat16, float16" : c10::toString(only)) + " with unit column stride"};
}

// Address of a packed device tensor of this shape; None: none.
void* packed(PyObject* o, const char* name, at::IntArrayRef shape, at::ScalarType type = at::kFloat) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() == type && t.is_cuda() && t.layout() == at::kStrided && t.sizes() == shape && t.is_contiguous()) return t.data_ptr();
    std::ostringstream why;
    why << name << " must be a packed device tensor of " << c10::toString(type) << " and shape " << shape;
    throw Refused{why.str()};
}
float* floats(PyObject* o, const char* name, at::IntArrayRef shape) { return (float*)packed(o, name, shape); }

struct Workspace {
    void* p = nullptr;
    size_t bytes = 0;
    explicit Workspace(PyObject* o) {
        if (o == Py_None) return;
        const at::Tensor& t = tensor(o, "workspace");
        if (!t.is_cuda() || t.layout() != at::kStrided || !t.is_contiguous()) throw Refused{"workspace must be a packed device tensor"};
        p = t.data_ptr();
        bytes = t.nbytes();
    }
};

struct Labels {
    void* p = nullptr;
    int32_t bits = 64;
    Labels(PyObject* o, int64_t n) {
        if (o == Py_None) return;
        const at::ScalarType type = tensor(o, "labels").scalar_type();
        if (type != at::kInt && type != at::kLong) throw Refused{"labels must be int32 or int64"};
        bits = type == at::kInt ? 32 : 64;
        p = packed(o, "labels", {n}, type);
    }
};

struct Kept {  // an 8-bit checkpoint
    Matrix q, e;
    Kept(PyObject* Q, PyObject* E) : q(matrix(Q, "Q", at::kChar)), e(matrix(E, "E", at::kByte)) {
        if (e.rows != q.rows || e.cols != (q.cols + 31) / 32) throw Refused{"E must have a row for each of Q's and a column for each 32 of Q's"};
    }
    const int8_t* codes() const { return (const int8_t*)q.p; }
    const uint8_t* steps() const { return (const uint8_t*)e.p; }
    void goes_with(const Matrix& x, const char* why) const {
        if (x.rows != q.rows || x.cols != q.cols) throw Refused{why};
    }
};
void alike(const Matrix& a, const Matrix& b, const char* why) {
    if (!a.alike(b)) throw Refused{why};
}

void* stream_of(PyObject* o) {
    void* p = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) throw python_error();
    return p;
}

// f(arguments) with the status of its call as the result, without the interpreter's lock while it enqueues.  The last argument is the raw stream.
template <int ARGUMENTS, class F>
PyObject* call(PyObject* const* a, Py_ssize_t count, F&& f) {
    if (count != ARGUMENTS) {
        PyErr_Format(PyExc_TypeError, "takes %d arguments, got %zd", ARGUMENTS, count);
        return nullptr;
    }
    try {
        auto enqueue = f(a, stream_of(a[ARGUMENTS - 1]));
        cbm_status status;
        Py_BEGIN_ALLOW_THREADS
        status = enqueue();
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    } catch (const Refused& r) {
        PyErr_SetString(PyExc_ValueError, r.why.c_str());
    } catch (python_error& e) {  // (the interpreter has it already)
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

PyObject* layer_norm(PyObject*, PyObject* const* args, Py_ssize_t count) {  // X, gamma, beta, eps, Y, mean, rstd, stream
    return call<8>(args, count, [](PyObject* const* a, void* stream) {
        const Matrix x = matrix(a[0], "X"), y = matrix(a[4], "Y");
        alike(x, y, "X and Y must have the same shape and type");
        const double eps = PyFloat_AsDouble(a[3]);
        if (PyErr_Occurred()) throw python_error();
        float *gamma = floats(a[1], "gamma", {x.cols}), *beta = floats(a[2], "beta", {x.cols}), *mean = floats(a[5], "mean", {x.rows}), *rstd = floats(a[6], "rstd", {x.rows});
        return [=] { return cbm_layer_norm(x.rows, columns(x.cols), x.type, x.p, x.ld, gamma, beta, (float)eps, y.p, y.ld, mean, rstd, stream); };
    });
}

PyObject* layer_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t count) {  // dY, X, gamma, mean, rstd, dX, dgamma, dbeta, workspace, stream
    return call<10>(args, count, [](PyObject* const* a, void* stream) {
        const Matrix g = matrix(a[0], "dY"), x = matrix(a[1], "X");
        alike(g, x, "dY and X must have the same shape and type");
        Matrix d{nullptr, x.cols, x.rows, x.cols, x.type};
        if (a[5] != Py_None) d = matrix(a[5], "dX");
        alike(g, d, "dY and dX must have the same shape and type");
        float *gamma = floats(a[2], "gamma", {x.cols}), *mean = floats(a[3], "mean", {x.rows}), *rstd = floats(a[4], "rstd", {x.rows});
        float *dgamma = floats(a[6], "dgamma", {x.cols}), *dbeta = floats(a[7], "dbeta", {x.cols});
        const Workspace w(a[8]);
        return [=] {
            return cbm_layer_norm_backward(x.rows, columns(x.cols), x.type, g.p, g.ld, x.p, x.ld, gamma, mean, rstd, d.p, d.ld, dgamma, dbeta, w.p, w.bytes, stream);
        };
    });
}

PyObject* checkpoint_save(PyObject*, PyObject* const* args, Py_ssize_t count) {  // X, Q, E, stream
    return call<4>(args, count, [](PyObject* const* a, void* stream) {
        const Matrix x = matrix(a[0], "X");
        const Kept k(a[1], a[2]);
        k.goes_with(x, "X and Q must have the same shape");
        return [=] { return cbm_checkpoint_save(x.rows, columns(x.cols), x.type, x.p, x.ld, (int8_t*)k.q.p, k.q.ld, (uint8_t*)k.e.p, k.e.ld, stream); };
    });
}

PyObject* checkpoint_restore(PyObject*, PyObject* const* args, Py_ssize_t count) {  // Q, E, X, stream
    return call<4>(args, count, [](PyObject* const* a, void* stream) {
        const Kept k(a[0], a[1]);
        const Matrix x = matrix(a[2], "X");
        k.goes_with(x, "X and Q must have the same shape");
        return [=] { return cbm_checkpoint_restore(x.rows, columns(x.cols), k.codes(), k.q.ld, k.steps(), k.e.ld, x.type, x.p, x.ld, stream); };
    });
}

PyObject* checkpoint_relu_backward(PyObject*, PyObject* const* args, Py_ssize_t count) {  // Q, E, dY, dX, stream
    return call<5>(args, count, [](PyObject* const* a, void* stream) {
        const Kept k(a[0], a[1]);
        const Matrix g = matrix(a[2], "dY"), d = matrix(a[3], "dX");
        alike(g, d, "dY and dX must have the same shape and type");
        k.goes_with(g, "dY and Q must have the same shape");
        return [=] { return cbm_checkpoint_relu_backward(g.rows, columns(g.cols), k.codes(), k.q.ld, k.steps(), k.e.ld, g.type, g.p, g.ld, d.p, d.ld, stream); };
    });
}

PyObject* checkpoint_weight_grad(PyObject*, PyObject* const* args, Py_ssize_t count) {  // Q, E, dY, dW, workspace, stream
    return call<6>(args, count, [](PyObject* const* a, void* stream) {
        const Kept k(a[0], a[1]);
        const Matrix g = matrix(a[2], "dY"), d = matrix(a[3], "dW", at::kFloat);
        if (g.rows != k.q.rows || d.rows != k.q.cols || d.cols != g.cols) throw Refused{"shape mismatch"};
        const Workspace w(a[4]);
        return [=] {
            return cbm_checkpoint_weight_grad(k.q.rows, columns(k.q.cols), columns(g.cols), k.codes(), k.q.ld, k.steps(), k.e.ld, g.type, g.p, g.ld, (float*)d.p, d.ld, w.p, w.bytes, stream);
        };
    });
}

PyObject* log_probs(PyObject*, PyObject* const* args, Py_ssize_t count) {  // Z, labels, logp, entropy, stats, top_values, top_columns, workspace, stream
    return call<9>(args, count, [](PyObject* const* a, void* stream) {
        const Matrix z = matrix(a[0], "Z");
        const Labels labels(a[1], z.rows);
        int64_t top = 0;
        if (a[5] != Py_None || a[6] != Py_None) {
            const at::Tensor& t = a[5] != Py_None ? tensor(a[5], "top_values") : tensor(a[6], "top_columns");
            top = t.dim() ? t.size(-1) : 0;
        }
        float *values = nullptr, *logp = floats(a[2], "logp", {z.rows}), *entropy = floats(a[3], "entropy", {z.rows}), *stats = floats(a[4], "stats", {z.rows, 2});
        int32_t* best = nullptr;
        if (a[5] != Py_None || a[6] != Py_None) {
            values = floats(a[5], "top_values", {z.rows, top});
            best = (int32_t*)packed(a[6], "top_columns", {z.rows, top}, at::kInt);
        }
        const Workspace w(a[7]);
        return [=] {
            return cbm_log_probs(z.rows, columns(z.cols), z.type, z.p, z.ld, labels.p, labels.bits, logp, entropy, stats, columns(top), values, best, w.p, w.bytes, stream);
        };
    });
}

PyObject* log_probs_backward(PyObject*, PyObject* const* args, Py_ssize_t count) {  // Z, labels, stats, entropy, dlogp, dentropy, dZ, stream
    return call<8>(args, count, [](PyObject* const* a, void* stream) {
        const Matrix z = matrix(a[0], "Z"), d = matrix(a[6], "dZ");
        alike(z, d, "Z and dZ must have the same shape and type");
        const Labels labels(a[1], z.rows);
        const float *stats = floats(a[2], "stats", {z.rows, 2}), *entropy = floats(a[3], "entropy", {z.rows}), *dlogp = floats(a[4], "dlogp", {z.rows}),
                    *dentropy = floats(a[5], "dentropy", {z.rows});
        return [=] { return cbm_log_probs_backward(z.rows, columns(z.cols), z.type, z.p, z.ld, labels.p, labels.bits, stats, entropy, dlogp, dentropy, d.p, d.ld, stream); };
    });
}

#define CBM_METHOD(name) {#name, (PyCFunction)(void (*)())name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CBM_METHOD(layer_norm), CBM_METHOD(layer_norm_backward), CBM_METHOD(checkpoint_save), CBM_METHOD(checkpoint_restore), CBM_METHOD(checkpoint_relu_backward),
                         CBM_METHOD(checkpoint_weight_grad), CBM_METHOD(log_probs), CBM_METHOD(log_probs_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) Py_CLEAR(m);  // whose layouts of tensors it reads
    return m;
}

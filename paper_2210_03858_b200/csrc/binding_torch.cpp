// CPython entry points that take and return torch tensors: the calls around a model's linears (logits, losses, microscaled
// matrices), which allocate their results.
//
// A call's GPU side can be as short as 6 us.  Checks and allocations written in Python took 12 to 19 us of the host (a
// tensor's attribute 0.1 us, an allocation 1.5, of which some calls make four); here they take 4 to 6, most of it the launch.
// The computation is behind the C ABI (include/bcq.h); load() resolves it from the library that is already loaded.  An
// operand that cannot be passed on raises ValueError or TypeError; a status other than BCQ_OK is returned as an int, which the
// Python side turns into its own error.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <exception>

#include "../../include/bcq.h"

namespace {

decltype(&bcq_token_logprobs) f_token_logprobs;
decltype(&bcq_distill_loss) f_distill_loss;
decltype(&bcq_distill_grad) f_distill_grad;
decltype(&bcq_mx_quantize) f_mx_quantize;
decltype(&bcq_mx_dequantize) f_mx_dequantize;
decltype(&bcq_mx_linear) f_mx_linear;

// An error whose Python form has been set.
struct Raised {};

[[noreturn]] void raise(PyObject* type, const char* format, const char* name, const char* more = "") {
    PyErr_Format(type, format, name, more);
    throw Raised();
}

// A tensor argument on the current device (the stream is that device's).
const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s must be a tensor", name);
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != c10::cuda::current_device()) raise(PyExc_ValueError, "%s must be on the current CUDA device", name);
    if (t.layout() != at::kStrided) raise(PyExc_TypeError, "%s must be a dense tensor", name);
    return t;
}
const at::Tensor& typed(PyObject* o, const char* name, at::ScalarType type) {
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != type) raise(PyExc_TypeError, "%s must be %s", name, c10::toString(type));
    return t;
}
const at::Tensor& dense(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape) {
    const at::Tensor& t = typed(o, name, type);
    if (t.sizes() != shape || !t.is_contiguous()) raise(PyExc_ValueError, "%s must be contiguous and have the shape that the other arguments give it", name);
    return t;
}

// Rows, columns and row pitch of a matrix whose rows are dense.
struct Rows {
    int n, cols, dtype;
    size_t ld;
};
Rows rows_of(const at::Tensor& t, const char* name) {
    if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) raise(PyExc_ValueError, "%s must have two dimensions and dense rows", name);
    if (t.size(0) > INT_MAX || t.size(1) > INT_MAX) raise(PyExc_ValueError, "%s is too large", name);
    Rows r;
    r.n = (int)t.size(0);
    r.cols = (int)t.size(1);
    r.ld = (size_t)(r.n > 1 ? t.stride(0) : std::max<int64_t>(t.size(1), t.stride(0)));
    if (t.scalar_type() == at::kFloat) r.dtype = BCQ_F32;
    else if (t.scalar_type() == at::kBFloat16) r.dtype = BCQ_BF16;
    else raise(PyExc_TypeError, "%s must be float32 or bfloat16", name);
    return r;
}

at::Tensor empty(at::IntArrayRef shape, at::ScalarType type) {
    return at::detail::empty_cuda(shape, type, c10::Device(c10::kCUDA, c10::cuda::current_device()), std::nullopt);
}

long as_int(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised();
    if (v > INT_MAX || v < INT_MIN) raise(PyExc_OverflowError, "%s is out of range", "an integer argument");
    return v;
}
float as_float(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return (float)v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised();
    return v != 0;
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }
template <typename T = void>
T* ptr(const at::Tensor& t) { return static_cast<T*>(t.data_ptr()); }

template <typename F>
int without_gil(F f) {
    PyThreadState* state = PyEval_SaveThread();
    const int st = f();
    PyEval_RestoreThread(state);
    return st;
}

PyObject* wrap(at::Tensor t) {
    PyObject* o = THPVariable_Wrap(std::move(t));
    if (o == nullptr) throw Raised();
    return o;
}
PyObject* tuple(std::initializer_list<PyObject*> items) {  // takes the references
    PyObject* t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject* o : items) {
        if (t != nullptr) PyTuple_SET_ITEM(t, i++, o);
        else Py_DECREF(o);
    }
    if (t == nullptr) throw Raised();
    return t;
}

// Nothing thrown leaves a call.
template <typename F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
        return nullptr;
    }
    try {
        return f();
    } catch (const Raised&) {
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// (logits, targets or None, top_k, temperature) -> (logprob or None, entropy, top_logprob, top_index)
PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 4, [&]() -> PyObject* {
        const at::Tensor& logits = tensor(a[0], "logits");
        const Rows r = rows_of(logits, "logits");
        const bool given = a[1] != Py_None;
        const at::Tensor* targets = given ? &dense(a[1], "targets", at::kLong, {r.n}) : nullptr;
        const int top_k = (int)as_int(a[2]);
        const float temperature = as_float(a[3]);
        // (without rows it only looks at sizes: a list that is refused is not allocated)
        const int fine = f_token_logprobs(0, r.cols, nullptr, r.ld, r.dtype, nullptr, top_k, temperature, nullptr, nullptr, nullptr, nullptr, nullptr);
        if (fine != BCQ_OK) return PyLong_FromLong(fine);
        at::Tensor logprob;
        if (given) logprob = empty({r.n}, at::kFloat);
        at::Tensor entropy = empty({r.n}, at::kFloat), top = empty({r.n, top_k}, at::kFloat), index = empty({r.n, top_k}, at::kInt);
        const int st = without_gil([&] {
            return f_token_logprobs(r.n, r.cols, ptr(logits), r.ld, r.dtype, given ? ptr<const long long>(*targets) : nullptr, top_k, temperature,
                                    given ? ptr<float>(logprob) : nullptr, ptr<float>(entropy), ptr<float>(top), ptr<int>(index), stream());
        });
        if (st != BCQ_OK) return PyLong_FromLong(st);
        PyObject* first = given ? wrap(logprob) : Py_NewRef(Py_None);
        return tuple({first, wrap(entropy), wrap(top), wrap(index)});
    });
}

struct Student {
    const at::Tensor& logits;
    Rows r;
    const at::Tensor &index, &logp;
    int k;
    explicit Student(PyObject* const* a)
        : logits(tensor(a[0], "logits")), r(rows_of(logits, "logits")), index(typed(a[1], "top_index", at::kInt)), logp(typed(a[2], "top_logprob", at::kFloat)) {
        if (index.dim() != 2 || index.size(0) != r.n || index.size(1) > INT_MAX || !index.is_contiguous())
            raise(PyExc_ValueError, "%s must be contiguous, with a row for each row of the logits", "top_index");
        if (logp.sizes() != index.sizes() || !logp.is_contiguous()) raise(PyExc_ValueError, "%s must be contiguous, of the shape of top_index", "top_logprob");
        k = (int)index.size(1);
    }
};

// (logits, top_index, top_logprob, temperature, tail) -> loss
PyObject* distill_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> PyObject* {
        const Student s(a);
        const float temperature = as_float(a[3]);
        const bool tail = truth(a[4]);
        at::Tensor loss = empty({s.r.n}, at::kFloat);
        const int st = without_gil([&] {
            return f_distill_loss(s.r.n, s.r.cols, s.k, ptr(s.logits), s.r.ld, s.r.dtype, ptr<int>(s.index), ptr<float>(s.logp), temperature, tail,
                                  ptr<float>(loss), stream());
        });
        return st != BCQ_OK ? PyLong_FromLong(st) : wrap(loss);
    });
}

// (logits, top_index, top_logprob, dloss, temperature, tail, out or None) -> (loss, dlogits)
PyObject* distill_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&]() -> PyObject* {
        const Student s(a);
        const at::Tensor& dloss = dense(a[3], "dloss", at::kFloat, {s.r.n});
        const float temperature = as_float(a[4]);
        const bool tail = truth(a[5]);
        at::Tensor out;
        if (a[6] == Py_None) {
            const int64_t pitch = ((int64_t)s.r.cols + 7) / 8 * 8;
            out = empty({s.r.n, pitch}, s.logits.scalar_type());
            if (pitch != s.r.cols) out = out.as_strided({s.r.n, s.r.cols}, {pitch, 1});
        } else {
            out = typed(a[6], "out", s.logits.scalar_type());
            if (out.sizes() != s.logits.sizes()) raise(PyExc_ValueError, "%s must have the shape of the logits", "out");
        }
        const Rows ro = rows_of(out, "out");
        at::Tensor loss = empty({s.r.n}, at::kFloat);
        const int st = without_gil([&] {
            return f_distill_grad(s.r.n, s.r.cols, s.k, ptr(s.logits), s.r.ld, s.r.dtype, ptr<int>(s.index), ptr<float>(s.logp), temperature, tail,
                                  ptr<float>(dloss), ptr<float>(loss), ptr(out), ro.ld, stream());
        });
        if (st != BCQ_OK) return PyLong_FromLong(st);
        PyObject* first = wrap(loss);
        return tuple({first, a[6] == Py_None ? wrap(out) : Py_NewRef(a[6])});
    });
}

// X -> (codes, scales, rows, cols)
PyObject* mx_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 1, [&]() -> PyObject* {
        const at::Tensor& X = tensor(a[0], "X");
        const Rows r = rows_of(X, "X");
        const int64_t atoms = ((int64_t)r.cols + 127) / 128;
        at::Tensor codes = empty({r.n, 64 * atoms}, at::kByte), scales = empty({((int64_t)r.n + 127) / 128, atoms, 32, 4, 4}, at::kByte);
        const int st = without_gil([&] { return f_mx_quantize(r.n, r.cols, ptr(X), r.ld, r.dtype, ptr<uint8_t>(codes), ptr<uint8_t>(scales), stream()); });
        if (st != BCQ_OK) return PyLong_FromLong(st);
        PyObject* first = wrap(codes);
        return tuple({first, wrap(scales), PyLong_FromLong(r.n), PyLong_FromLong(r.cols)});
    });
}

struct Mx {
    const at::Tensor &codes, &scales;
    int rows, cols;
    // codes, scales, rows, cols
    Mx(PyObject* const* a, const char* name)
        : codes(typed(a[0], name, at::kByte)), scales(typed(a[1], name, at::kByte)), rows((int)as_int(a[2])), cols((int)as_int(a[3])) {
        if (rows < 0 || cols < 1) raise(PyExc_ValueError, "%s must have at least 0 rows and 1 column", name);
        const int64_t atoms = ((int64_t)cols + 127) / 128;
        if (codes.sizes() != at::IntArrayRef({rows, 64 * atoms}) || !codes.is_contiguous() ||
            scales.sizes() != at::IntArrayRef({((int64_t)rows + 127) / 128, atoms, 32, 4, 4}) || !scales.is_contiguous())
            raise(PyExc_ValueError, "%s: codes and scales must be contiguous, of shapes [rows][64 * ceil(cols / 128)] and "
                                    "[ceil(rows / 128)][ceil(cols / 128)][32][4][4]", name);
    }
};

// (codes, scales, rows, cols) -> None
PyObject* mx_check(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 4, [&]() -> PyObject* {
        const Mx m(a, "an MxMatrix");
        (void)m;
        return Py_NewRef(Py_None);
    });
}

// (codes, scales, rows, cols, bf16) -> values
PyObject* mx_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> PyObject* {
        const Mx m(a, "M");
        const bool bf16 = truth(a[4]);
        at::Tensor out = empty({m.rows, m.cols}, bf16 ? at::kBFloat16 : at::kFloat);
        const int st = without_gil([&] {
            return f_mx_dequantize(m.rows, m.cols, ptr<uint8_t>(m.codes), ptr<uint8_t>(m.scales), ptr(out), (size_t)m.cols, bf16 ? BCQ_BF16 : BCQ_F32, stream());
        });
        return st != BCQ_OK ? PyLong_FromLong(st) : wrap(out);
    });
}

// (X's codes, scales, rows, cols, W's codes, scales, rows, cols, bias or None, out or None, bf16) -> Y
PyObject* mx_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&]() -> PyObject* {
        const Mx X(a, "X"), W(a + 4, "W");
        if (X.cols != W.cols) raise(PyExc_ValueError, "%s and W must have the same number of columns", "X");
        const bool biased = a[8] != Py_None;
        const at::Tensor* bias = biased ? &dense(a[8], "bias", at::kFloat, {W.rows}) : nullptr;
        at::Tensor out;
        if (a[9] == Py_None) {
            out = empty({X.rows, W.rows}, truth(a[10]) ? at::kBFloat16 : at::kFloat);
        } else {
            out = tensor(a[9], "out");
            if (out.sizes() != at::IntArrayRef({X.rows, W.rows})) raise(PyExc_ValueError, "%s must have a row for each of X's and a column for each of W's rows", "out");
        }
        const Rows ro = rows_of(out, "out");
        const int st = without_gil([&] {
            return f_mx_linear(W.rows, W.cols, X.rows, ptr<uint8_t>(X.codes), ptr<uint8_t>(X.scales), ptr<uint8_t>(W.codes), ptr<uint8_t>(W.scales),
                               biased ? ptr<float>(*bias) : nullptr, ptr(out), ro.ld, ro.dtype, stream());
        });
        if (st != BCQ_OK) return PyLong_FromLong(st);
        return a[9] == Py_None ? wrap(out) : Py_NewRef(a[9]);
    });
}

PyObject* load(PyObject*, PyObject* path) {
    const char* file = PyUnicode_AsUTF8(path);
    if (file == nullptr) return nullptr;
    void* h = dlopen(file, RTLD_NOW);
    if (h == nullptr) {
        PyErr_SetString(PyExc_RuntimeError, dlerror());
        return nullptr;
    }
    const struct {
        const char* name;
        void** slot;
    } table[] = {
        {"bcq_token_logprobs", (void**)&f_token_logprobs}, {"bcq_distill_loss", (void**)&f_distill_loss}, {"bcq_distill_grad", (void**)&f_distill_grad},
        {"bcq_mx_quantize", (void**)&f_mx_quantize}, {"bcq_mx_dequantize", (void**)&f_mx_dequantize}, {"bcq_mx_linear", (void**)&f_mx_linear},
    };
    for (const auto& e : table) {
        void* sym = dlsym(h, e.name);
        if (sym == nullptr) {
            PyErr_Format(PyExc_RuntimeError, "%s is missing from %s", e.name, file);
            return nullptr;
        }
        *e.slot = sym;
    }
    Py_RETURN_NONE;
}

#define M(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {M(token_logprobs), M(distill_loss), M(distill_grad), M(mx_quantize), M(mx_check), M(mx_dequantize), M(mx_linear),
                         {"load", load, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_call(void) { return PyModule_Create(&module); }

// Python's side of the calls of a serving step (the router, products, norm, quantisation, combination): takes tensors apart,
// checks what the C library cannot see -- element types, shapes, strides, that they are on one GPU -- and calls it.  A call
// of binding.py by ctypes takes 6 us for this, as long as the kernel of a small step; here it is under one.  Every function
// takes its arguments by position, None for what is not given, the stream's address last, and returns the C function's
// code; what does not fit raises ValueError.
#include <Python.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdexcept>
#include <string>

#include "csr5.h"

namespace {

struct Refused : std::runtime_error {
    using std::runtime_error::runtime_error;
};

struct Raised {};       // Python's exception is set

struct Matrix {
    void* p = nullptr;
    int64_t rows = 0, cols = 0, ld = 0, group = 0, groups = 0;
    at::ScalarType type = at::kFloat;
};

bool is_f8(at::ScalarType t) { return t == at::kFloat8_e4m3fn || t == at::kByte; }

int code(at::ScalarType t, const char* name) {
    if (t == at::kBFloat16) return CSR5_DTYPE_BF16;
    if (t == at::kHalf) return CSR5_DTYPE_F16;
    if (t == at::kFloat) return CSR5_DTYPE_F32;
    throw Refused(std::string(name) + ": expected dtype bfloat16, float16 or float32, got " + at::toString(t));
}

std::string shape_text(std::initializer_list<int64_t> dims) {
    std::string s = "(";
    for (int64_t d : dims) s += (s.size() > 1 ? ", " : "") + (d < 0 ? std::string("any") : std::to_string(d));
    return s + ")";
}

// The arguments of a call.
class Args {
public:
    Args(PyObject* const* a, Py_ssize_t n, Py_ssize_t want) : a_(a) {
        if (n != want) throw Refused("expected " + std::to_string(want) + " arguments, got " + std::to_string(n));
    }
    bool none(int i) const { return a_[i] == Py_None; }
    const at::Tensor& tensor(int i, const char* name) const {
        if (!THPVariable_Check(a_[i])) throw Refused(std::string(name) + ": expected a tensor");
        const at::Tensor& t = THPVariable_Unpack(a_[i]);
        const at::ScalarType s = t.scalar_type();
        if (!is_f8(s) && s != at::kInt) code(s, name);          // a type of none of these calls is what to say first
        if (!t.is_cuda()) throw Refused(std::string(name) + ": expected a GPU tensor");
        const int gpu = t.get_device();
        if (gpu_ >= 0 && gpu != gpu_) throw Refused(std::string(name) + ": expected a tensor on GPU " + std::to_string(gpu_) + " as the others, got one on GPU " + std::to_string(gpu));
        gpu_ = gpu;
        return t;
    }
    int32_t number(int i, const char* name) const {
        const long v = PyLong_AsLong(a_[i]);
        if ((v == -1 && PyErr_Occurred()) || v != int32_t(v)) {
            PyErr_Clear();
            throw Refused(std::string(name) + ": expected a 32-bit whole number");
        }
        return int32_t(v);
    }
    double real(int i, const char* name) const {
        const double v = PyFloat_AsDouble(a_[i]);
        if (v == -1.0 && PyErr_Occurred()) {
            PyErr_Clear();
            throw Refused(std::string(name) + ": expected a number");
        }
        return v;
    }
    // the stream: its address, a torch stream, or None: torch's current one.  In a statement of its own after all others (arguments
    // of a call are evaluated in any order), as it may have to make the device ready.  Refused where it is of another GPU than the
    // tensors (which an address does not say).
    void* stream(int i) const {
        PyObject* at = a_[i];
        PyObject* own = nullptr;
        int gpu = gpu_;
        if (at == Py_None) {
            at = own = PyObject_CallObject(current_stream, nullptr);
            if (at) gpu = c10::impl::VirtualGuardImpl(at::kCUDA).getDevice().index();
        } else if (!PyLong_Check(at)) {
            PyObject* const index = PyObject_GetAttrString(at, "device_index");
            if (index) gpu = int(PyLong_AsLong(index));
            Py_XDECREF(index);
            PyErr_Clear();
            at = own = PyObject_GetAttrString(at, "cuda_stream");
        }
        if (!at) throw Raised();
        void* const p = at == Py_None ? nullptr : PyLong_AsVoidPtr(at);
        Py_XDECREF(own);
        if (!p && PyErr_Occurred()) throw Raised();
        if (gpu != gpu_) throw Refused("the tensors are on GPU " + std::to_string(gpu_) + ", the stream is one of GPU " + std::to_string(gpu));
        return p;
    }
    static PyObject* current_stream;        // returns the current stream's address

    // Rows that are contiguous; 3-D where `groups` (given, or any: -1) is not 0.  rows, cols: given, or any: -1.
    Matrix matrix(int i, const char* name, int64_t rows = -1, int64_t cols = -1, int64_t groups = 0) const {
        const at::Tensor& t = tensor(i, name);
        const int d = groups != 0;
        Matrix m;
        m.type = t.scalar_type();
        const bool fits = t.dim() == 2 + d && (!d || groups < 0 || t.size(0) == groups) && (rows < 0 || t.size(d) == rows) && (cols < 0 || t.size(d + 1) == cols);
        if (!fits) {
            std::string got = "(";
            for (int64_t s : t.sizes()) got += (got.size() > 1 ? ", " : "") + std::to_string(s);
            throw Refused(std::string(name) + ": expected shape " + (d ? shape_text({groups, rows, cols}) : shape_text({rows, cols})) + ", got " + got + ")");
        }
        m.rows = t.size(d), m.cols = t.size(d + 1), m.groups = d ? t.size(0) : 1;
        if (m.rows != int32_t(m.rows) || m.cols != int32_t(m.cols) || m.groups != int32_t(m.groups)) throw Refused(std::string(name) + ": too large");
        if (t.stride(d + 1) != 1 && m.cols > 1) throw Refused(std::string(name) + ": expected a GPU tensor with contiguous rows");
        m.ld = m.rows > 1 ? t.stride(d) : std::max(t.stride(d), m.cols), m.group = d ? t.stride(0) : 0;
        m.p = t.data_ptr();
        return m;
    }
    Matrix typed(int i, const char* name, at::ScalarType type, int64_t rows, int64_t cols, int64_t groups = 0) const {
        const Matrix m = matrix(i, name, rows, cols, groups);
        if (m.type != type) throw Refused(std::string(name) + ": expected dtype " + at::toString(type) + ", got " + at::toString(m.type));
        return m;
    }
    Matrix maybe(int i, const char* name, at::ScalarType type, int64_t rows, int64_t cols) const { return none(i) ? Matrix() : typed(i, name, type, rows, cols); }
    Matrix f8(int i, const char* name, int64_t rows = -1, int64_t cols = -1, int64_t groups = 0) const {
        const Matrix m = matrix(i, name, rows, cols, groups);
        if (!is_f8(m.type)) throw Refused(std::string(name) + ": expected dtype float8_e4m3fn or uint8, got " + at::toString(m.type));
        return m;
    }
    // float32 scales in any layout; group, ld and cols: their strides
    Matrix scales(int i, const char* name, int64_t rows, int64_t blocks, int64_t groups = 0) const {
        const at::Tensor& t = tensor(i, name);
        const int d = groups != 0;
        if (t.scalar_type() != at::kFloat) throw Refused(std::string(name) + ": expected a float32 GPU tensor");
        if (t.dim() != 2 + d || (d && t.size(0) != groups) || t.size(d) != rows || t.size(d + 1) != blocks)
            throw Refused(std::string(name) + ": expected shape " + (d ? shape_text({groups, rows, blocks}) : shape_text({rows, blocks})));
        Matrix m;
        m.p = t.data_ptr(), m.ld = t.stride(d), m.cols = t.stride(d + 1), m.group = d ? t.stride(0) : 0;
        return m;
    }
    // at least `least` contiguous values
    template <typename V> V* array(int i, const char* name, at::ScalarType type, int64_t least) const {
        if (none(i)) return nullptr;
        const at::Tensor& t = tensor(i, name);
        if (t.scalar_type() != type) throw Refused(std::string(name) + ": expected dtype " + at::toString(type) + ", got " + at::toString(t.scalar_type()));
        if (t.numel() < least) throw Refused(std::string(name) + ": needs at least " + std::to_string(least) + " elements, has " + std::to_string(t.numel()));
        if (!t.is_contiguous()) throw Refused(std::string(name) + ": expected a contiguous GPU tensor");
        return static_cast<V*>(t.data_ptr());
    }
    int32_t* whole(int i, const char* name, int64_t least) const { return array<int32_t>(i, name, at::kInt, least); }
    float* floats(int i, const char* name, int64_t least) const { return array<float>(i, name, at::kFloat, least); }
    // the source of `rows` rows, of x_rows
    int32_t* source(int i, int64_t rows, int64_t x_rows) const {
        if (none(i) && x_rows < rows) throw Refused("x: needs " + std::to_string(rows) + " rows without source, has " + std::to_string(x_rows));
        return whole(i, "source", rows);
    }

private:
    PyObject* const* a_;
    mutable int gpu_ = -1;      // of the tensors so far
};

PyObject* Args::current_stream = nullptr;

int64_t blocks(int64_t n) { return (n + CSR5_F8_BLOCK - 1) / CSR5_F8_BLOCK; }
template <typename T> T* as(const Matrix& m) { return static_cast<T*>(m.p); }

// logits, k, expert, weight, offset, source, place, workspace, stream
int route(const Args& a) {
    const Matrix l = a.matrix(0, "logits");
    const int dtype = code(l.type, "logits");
    const int32_t k = a.number(1, "k");
    const int64_t pairs = l.rows * std::max(k, 0);
    uint8_t* const space = a.array<uint8_t>(7, "workspace", at::kByte, 0);
    const size_t bytes = a.none(7) ? 0 : size_t(a.tensor(7, "workspace").numel());
    int32_t *const expert = a.whole(2, "expert", pairs), *const offset = a.whole(4, "offset", l.cols + 1);
    int32_t *const source = a.whole(5, "source", pairs), *const place = a.whole(6, "place", pairs);
    float* const weight = a.floats(3, "weight", pairs);
    void* const stream = a.stream(8);
    return csr5_route(int32_t(l.rows), int32_t(l.cols), k, dtype, l.p, l.ld, expert, weight, offset, source, place, space, bytes, stream);
}

// z, place, y, weight, residual, stream
int combine(const Args& a) {
    const Matrix z = a.matrix(0, "z");
    const int dtype = code(z.type, "z");
    const at::Tensor& place = a.tensor(1, "place");
    if (place.dim() != 2) throw Refused("place: expected a 2-D tensor");
    const int64_t tokens = place.size(0), k = place.size(1);
    if (tokens != int32_t(tokens) || k != int32_t(k)) throw Refused("place: too large");
    const Matrix y = a.typed(2, "y", z.type, tokens, z.cols), r = a.maybe(4, "residual", z.type, tokens, z.cols);
    const int32_t* const row = a.whole(1, "place", tokens * k);
    const float* const weight = a.floats(3, "weight", tokens * k);
    void* const stream = a.stream(5);
    return csr5_combine(int32_t(tokens), int32_t(k), int32_t(z.rows), int32_t(z.cols), dtype, z.p, z.ld, row, weight, r.p, r.ld, y.p, y.ld, stream);
}

// x, w, offset, y, source, stream
int grouped_gemm(const Args& a) {
    const Matrix x = a.matrix(0, "x");
    const int dtype = code(x.type, "x");
    const Matrix w = a.typed(1, "w", x.type, -1, x.cols, -1), y = a.typed(3, "y", x.type, -1, w.rows);
    const int32_t *const offset = a.whole(2, "offset", w.groups + 1), *const source = a.source(4, y.rows, x.rows);
    void* const stream = a.stream(5);
    return csr5_grouped_gemm(int32_t(w.groups), int32_t(y.rows), int32_t(w.rows), int32_t(x.cols), dtype, offset, x.p, int32_t(x.rows), x.ld, source, w.p, w.ld, w.group, y.p,
                             y.ld, stream);
}

// x, q, scale, block_rows, stream
int quantise(const Args& a) {
    const Matrix x = a.matrix(0, "x");
    const int dtype = code(x.type, "x");
    const int32_t by = a.number(3, "block_rows");
    const Matrix q = a.f8(1, "q", x.rows, x.cols), s = a.scales(2, "scale", by > 0 ? (x.rows + by - 1) / by : 0, blocks(x.cols));
    void* const stream = a.stream(4);
    return csr5_quantise(int32_t(x.rows), int32_t(x.cols), by, dtype, x.p, x.ld, as<uint8_t>(q), q.ld, as<float>(s), s.ld, s.cols, stream);
}

// x, x_scale, w, w_scale, y, w_rows, stream
int gemm_f8(const Args& a) {
    const Matrix x = a.f8(0, "x"), w = a.f8(2, "w", -1, x.cols), y = a.matrix(4, "y", x.rows, w.rows);
    const int dtype = code(y.type, "y");
    const int32_t by = a.number(5, "w_rows");
    const Matrix xs = a.scales(1, "x_scale", x.rows, blocks(x.cols)), ws = a.scales(3, "w_scale", by > 0 ? (w.rows + by - 1) / by : 0, blocks(x.cols));
    void* const stream = a.stream(6);
    return csr5_gemm_f8(int32_t(x.rows), int32_t(w.rows), int32_t(x.cols), dtype, as<uint8_t>(x), x.ld, as<float>(xs), xs.ld, xs.cols, as<uint8_t>(w), w.ld, as<float>(ws), by, ws.ld,
                        ws.cols, y.p, y.ld, stream);
}

// x, x_scale, w, w_scale, offset, y, w_rows, source, stream
int grouped_gemm_f8(const Args& a) {
    const Matrix x = a.f8(0, "x"), w = a.f8(2, "w", -1, x.cols, -1), y = a.matrix(5, "y", -1, w.rows);
    const int dtype = code(y.type, "y");
    const int32_t by = a.number(6, "w_rows");
    const Matrix xs = a.scales(1, "x_scale", x.rows, blocks(x.cols));
    if (w.groups == 0) return CSR5_OK;              // no scales to look at
    const Matrix ws = a.scales(3, "w_scale", by > 0 ? (w.rows + by - 1) / by : 0, blocks(x.cols), w.groups);
    const int32_t *const offset = a.whole(4, "offset", w.groups + 1), *const source = a.source(7, y.rows, x.rows);
    void* const stream = a.stream(8);
    return csr5_grouped_gemm_f8(int32_t(w.groups), int32_t(y.rows), int32_t(w.rows), int32_t(x.cols), dtype, offset, as<uint8_t>(x), int32_t(x.rows), x.ld, as<float>(xs), xs.ld,
                                xs.cols, source, as<uint8_t>(w), w.ld, w.group, as<float>(ws), by, ws.ld, ws.cols, ws.group, y.p, y.ld, stream);
}

// x, gain, eps, residual, h, y, q, scale, rstd, stream
int rmsnorm(const Args& a) {
    if (a.none(6) != a.none(7)) throw Refused("q and scale: both or neither");
    const Matrix x = a.matrix(0, "x");
    const int dtype = code(x.type, "x");
    const void* gain = nullptr;
    if (!a.none(1)) {
        const at::Tensor& g = a.tensor(1, "gain");
        if (g.scalar_type() != x.type || g.dim() != 1 || g.size(0) != x.cols || !g.is_contiguous())
            throw Refused("gain: expected a contiguous GPU tensor of " + std::to_string(x.cols) + " values of " + at::toString(x.type));
        gain = g.data_ptr();
    }
    const Matrix r = a.maybe(3, "residual", x.type, x.rows, x.cols), h = a.maybe(4, "h", x.type, x.rows, x.cols), y = a.maybe(5, "y", x.type, x.rows, x.cols);
    const Matrix q = a.none(6) ? Matrix() : a.f8(6, "q", x.rows, x.cols), s = a.none(7) ? Matrix() : a.scales(7, "scale", x.rows, blocks(x.cols));
    const float eps = float(a.real(2, "eps"));
    float* const rstd = a.floats(8, "rstd", x.rows);
    void* const stream = a.stream(9);
    return csr5_rmsnorm(int32_t(x.rows), int32_t(x.cols), dtype, x.p, x.ld, r.p, r.ld, gain, eps, h.p, h.ld, y.p, y.ld, as<uint8_t>(q), q.ld, as<float>(s), s.ld, s.cols, rstd, stream);
}

template <int (*F)(const Args&), int COUNT> PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        return PyLong_FromLong(F(Args(args, n, COUNT)));
    } catch (const Raised&) {
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

PyObject* set_current_stream(PyObject*, PyObject* f) {
    Py_INCREF(f);
    Py_XDECREF(Args::current_stream);
    Args::current_stream = f;
    Py_RETURN_NONE;
}

#define ENTRY(name, count) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(entry<name, count>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(route, 9), ENTRY(combine, 6), ENTRY(grouped_gemm, 6), ENTRY(quantise, 5), ENTRY(gemm_f8, 7), ENTRY(grouped_gemm_f8, 9), ENTRY(rmsnorm, 10), {"set_current_stream", set_current_stream, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }

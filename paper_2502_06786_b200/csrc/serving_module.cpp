// The Python side of the serving entry points: argument checks on torch tensors and the call, without ctypes.
//
// A decode step's call takes a few microseconds on the GPU.  Reading a dozen tensors' attributes from Python and converting eighteen arguments with
// ctypes takes ten; here it takes about one, and the launch itself is what is left.  The functions take positional arguments only and return the
// library's status; defaults, allocation of outputs and MatqError live in binding.py.
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>
#include <string>

#include "matq.h"

namespace {

struct Bad {
    PyObject* type;
    std::string what;
};
[[noreturn]] void fail(PyObject* type, const char* name, const char* what) { throw Bad{type, std::string(name) + ": " + what}; }

// a CUDA tensor on the current device, whose stream the call uses; of one type, if that matters (std::nullopt: any)
const at::Tensor& tensor(PyObject* o, std::optional<at::ScalarType> type, const char* name) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, name, "expected a CUDA tensor");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || (type && t.scalar_type() != *type))
        fail(PyExc_TypeError, name, (std::string("expected a CUDA tensor") + (type ? std::string(" of dtype ") + c10::toString(*type) : "")).c_str());
    if (t.get_device() != c10::cuda::current_device()) fail(PyExc_ValueError, name, "on another device than the current one, whose stream the call would use");
    return t;
}
template <typename T>
T* vec(PyObject* o, at::ScalarType type, const char* name, int64_t n) {
    const at::Tensor& t = tensor(o, type, name);
    if (t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1)) fail(PyExc_ValueError, name, (std::string("contiguous, ") + std::to_string(n) + " elements required").c_str());
    return static_cast<T*>(t.data_ptr());
}
struct Matrix {
    void* p;
    int64_t rows, cols, ld;
};
Matrix mat(PyObject* o, at::ScalarType type, const char* name) {
    const at::Tensor& t = tensor(o, type, name);
    if (t.dim() != 2) fail(PyExc_ValueError, name, "expected 2 dimensions");
    const int64_t r = t.size(0), c = t.size(1);
    if (t.stride(1) != 1 && c > 1) fail(PyExc_ValueError, name, "unit stride along its second dimension required");
    return {t.data_ptr(), r, c, r > 1 ? t.stride(0) : c};               // a single row may report any stride
}
struct Heads {
    void* p;
    int64_t T, H, ld;
};
Heads heads(PyObject* o, const char* name, int64_t D) {
    const at::Tensor& t = tensor(o, at::kBFloat16, name);
    if (t.dim() != 3) fail(PyExc_ValueError, name, "expected 3 dimensions");
    const int64_t T = t.size(0), H = t.size(1);
    if (t.size(2) != D || (t.stride(2) != 1 && D > 1) || (t.stride(1) != D && H > 1)) fail(PyExc_ValueError, name, "bf16 [T, heads, head_dim] with a token's heads adjacent required");
    return {t.data_ptr(), T, H, T > 1 ? t.stride(0) : H * D};
}
int32_t* status_word(PyObject* o) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, at::kInt, "dev_status");
    if (t.numel() < 1) fail(PyExc_ValueError, "dev_status", "one element required");
    return static_cast<int32_t*>(t.data_ptr());
}
int64_t integer(PyObject* o, const char* name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); fail(PyExc_TypeError, name, "an integer is required"); }
    return v;
}
int small_integer(PyObject* o, const char* name) {
    const int64_t v = integer(o, name);
    if (v < 0 || v > INT32_MAX) fail(PyExc_ValueError, name, "out of range");
    return (int)v;
}
double number(PyObject* o, const char* name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); fail(PyExc_TypeError, name, "a number is required"); }
    return v;
}
// Other Python threads run meanwhile: a launch waits while the stream's queue is full.  Nothing of Python is touched by f.
template <typename F>
int unlocked(F f) {
    PyThreadState* state = PyEval_SaveThread();
    const int st = f();
    PyEval_RestoreThread(state);
    return st;
}
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

struct Paged {
    matq_paged_kv c;
};
Paged paged(PyObject* const* a) {
    const at::Tensor &k = tensor(a[0], at::kBFloat16, "k_cache"), &v = tensor(a[1], at::kBFloat16, "v_cache");
    if (k.dim() != 4 || k.sizes() != v.sizes() || !k.is_contiguous() || !v.is_contiguous())
        fail(PyExc_ValueError, "k_cache, v_cache", "contiguous [n_pages, kv_heads, page_size, head_dim] of one shape required");
    if (k.size(1) > INT32_MAX || k.size(2) > INT32_MAX || k.size(3) > INT32_MAX) fail(PyExc_ValueError, "k_cache", "a dimension is too large");
    const Matrix t = mat(a[2], at::kInt, "page_table");
    if (t.rows > INT32_MAX - 1) fail(PyExc_ValueError, "page_table", "too many sequences");
    Paged p;
    p.c.k = k.data_ptr();
    p.c.v = v.data_ptr();
    p.c.n_pages = k.size(0);
    p.c.kv_heads = (int)k.size(1);
    p.c.page_size = (int)k.size(2);
    p.c.head_dim = (int)k.size(3);
    p.c.batch = (int)t.rows;
    p.c.page_table = static_cast<const int32_t*>(t.p);
    p.c.table_stride = t.ld;
    p.c.table_width = t.cols;
    p.c.cu_q = vec<int32_t>(a[3], at::kInt, "cu_q", t.rows + 1);
    p.c.kv_len = vec<int32_t>(a[4], at::kInt, "kv_len", t.rows);
    return p;
}

template <typename F>
PyObject* call(Py_ssize_t n, Py_ssize_t want, F f) {
    if (n != want) return PyErr_Format(PyExc_TypeError, "%zd positional arguments required, %zd given", want, n);
    try {
        return PyLong_FromLong(f());
    } catch (const Bad& b) {
        PyErr_SetString(b.type, b.what.c_str());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

// X, xq, scale, rowsum, dev_status
PyObject* quantize_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 5, [&] {
        const Matrix x = mat(a[0], at::kBFloat16, "X"), o = mat(a[1], at::kChar, "xq");
        if (o.rows != x.rows || o.cols != x.cols) fail(PyExc_ValueError, "xq", "int8 [M, K] required");
        float* scale = vec<float>(a[2], at::kFloat, "scale", x.rows);
        int32_t *rowsum = vec<int32_t>(a[3], at::kInt, "rowsum", x.rows), *status = status_word(a[4]);
        void* s = stream();
        return unlocked([&] { return matq_quantize_tokens(x.p, x.rows, x.cols, x.ld, static_cast<int8_t*>(o.p), o.ld, scale, rowsum, status, s); });
    });
}

// xq, scale, rowsum, q, alpha, zero, y, flags, dev_status, c
PyObject* gemm_a8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 10, [&] {
        const Matrix x = mat(a[0], at::kChar, "xq"), w = mat(a[3], at::kByte, "q");
        if (w.cols != x.cols) fail(PyExc_ValueError, "q", "xq [M, K] and q [N, K] required");
        const bool bf16 = THPVariable_Check(a[6]) && THPVariable_Unpack(a[6]).scalar_type() == at::kBFloat16;
        const Matrix y = mat(a[6], bf16 ? at::kBFloat16 : at::kFloat, "y");
        if (y.rows != x.rows || y.cols != w.rows) fail(PyExc_ValueError, "y", "[M, N] required");
        const float *scale = vec<float>(a[1], at::kFloat, "scale", x.rows), *alpha = vec<float>(a[4], at::kFloat, "alpha", w.rows),
                    *zero = vec<float>(a[5], at::kFloat, "zero", w.rows);
        const int32_t* rowsum = vec<int32_t>(a[2], at::kInt, "rowsum", x.rows);
        const int flags = small_integer(a[7], "flags"), c = small_integer(a[9], "c");
        int32_t* status = status_word(a[8]);
        void* s = stream();
        return unlocked([&] {
            return matq_gemm_a8(static_cast<const int8_t*>(x.p), x.rows, x.cols, x.ld, scale, rowsum, static_cast<const uint8_t*>(w.p), w.rows, w.ld, c, alpha, zero,
                                bf16 ? MATQ_OUT_BF16 : MATQ_OUT_F32, y.p, y.ld, (unsigned)flags, status, s);
        });
    });
}

// k_cache, v_cache, page_table, cu_q, kv_len, k, v, cos_sin, q, q_out, interleaved, dev_status
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 12, [&] {
        const Paged p = paged(a);
        const int64_t D = p.c.head_dim;
        const Heads k = heads(a[5], "k", D), v = heads(a[6], "v", D);
        if (k.H != p.c.kv_heads || v.H != p.c.kv_heads || v.T != k.T) fail(PyExc_ValueError, "k, v", "[T, kv_heads, head_dim] each required");
        Matrix cs = {nullptr, 0, 0, 0};
        if (a[7] != Py_None) {
            cs = mat(a[7], at::kFloat, "cos_sin");
            if (cs.ld != cs.cols) fail(PyExc_ValueError, "cos_sin", "contiguous [max_pos, rot_dim] required");
        }
        Heads q = {nullptr, 0, 0, 0}, o = q;
        if ((a[8] == Py_None) != (a[9] == Py_None)) fail(PyExc_ValueError, "q, q_out", "both or neither required");
        if (a[8] != Py_None) {
            q = heads(a[8], "q", D);
            o = heads(a[9], "q_out", D);
            if (q.T != k.T || o.T != k.T || q.H != o.H) fail(PyExc_ValueError, "q, q_out", "one row per token each, of the same heads");
        }
        const int inter = PyObject_IsTrue(a[10]);
        if (inter < 0) { PyErr_Clear(); fail(PyExc_TypeError, "interleaved", "a truth value is required"); }
        int32_t* status = status_word(a[11]);
        void* s = stream();
        return unlocked([&] {
            return matq_kv_append(&p.c, k.T, q.p, (int)q.H, q.ld, k.p, k.ld, v.p, v.ld, static_cast<const float*>(cs.p), cs.rows, (int)cs.cols, inter, o.p, o.ld, status, s);
        });
    });
}

// q, k_cache, v_cache, page_table, cu_q, kv_len, max_q, max_kv, scale, softcap, window, out, workspace, dev_status
PyObject* attn_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 14, [&] {
        const Paged p = paged(a + 1);
        const int64_t D = p.c.head_dim;
        const Heads q = heads(a[0], "q", D), o = heads(a[11], "out", D);
        if (o.T != q.T || o.H != q.H) fail(PyExc_ValueError, "out", "one row per token, of q's heads");
        void* ws = nullptr;
        size_t bytes = 0;
        if (a[12] != Py_None) {
            const at::Tensor& t = tensor(a[12], std::nullopt, "workspace");
            if (!t.is_contiguous()) fail(PyExc_TypeError, "workspace", "a contiguous tensor is required");
            ws = t.data_ptr();
            bytes = t.nbytes();
        }
        const float scale = (float)number(a[8], "scale"), softcap = (float)number(a[9], "softcap");
        const int64_t window = integer(a[10], "window"), max_q = integer(a[6], "max_q"), max_kv = integer(a[7], "max_kv");
        int32_t* status = status_word(a[13]);
        void* s = stream();
        return unlocked([&] { return matq_attn_paged(&p.c, q.T, q.p, (int)q.H, q.ld, scale, softcap, window, max_q, max_kv, o.p, o.ld, ws, bytes, status, s); });
    });
}

PyMethodDef methods[] = {
    {"quantize_tokens", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(quantize_tokens)), METH_FASTCALL, nullptr},
    {"gemm_a8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gemm_a8)), METH_FASTCALL, nullptr},
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_append)), METH_FASTCALL, nullptr},
    {"attn_paged", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attn_paged)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serving", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving(void) { return PyModule_Create(&module); }

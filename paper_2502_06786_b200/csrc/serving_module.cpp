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
bool is_bf16(PyObject* o) { return THPVariable_Check(o) && THPVariable_Unpack(o).scalar_type() == at::kBFloat16; }       // of an output of either type
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
    if (t.stride(1) != 1 && c > 1 && r > 0) fail(PyExc_ValueError, name, "unit stride along its second dimension required");
    return {t.data_ptr(), r, c, r > 1 ? t.stride(0) : c};               // a single row, or none, may report any stride
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

struct Paged4 {
    matq_paged_kv4 c;
};
Paged4 paged4(PyObject* const* a) {
    const at::Tensor& tiles = tensor(a[0], at::kByte, "cache");
    if (tiles.dim() != 4 || !tiles.is_contiguous()) fail(PyExc_ValueError, "cache", "contiguous [n_pages, kv_heads, page_size / 16, 18 head_dim] required");
    if (tiles.size(1) > INT32_MAX || tiles.size(2) > INT32_MAX / 16 || tiles.size(3) > INT32_MAX || tiles.size(3) % 18 != 0) fail(PyExc_ValueError, "cache", "[n_pages, kv_heads, page_size / 16, 18 head_dim] required");
    const Matrix t = mat(a[1], at::kInt, "page_table");
    if (t.rows > INT32_MAX - 1) fail(PyExc_ValueError, "page_table", "too many sequences");
    Paged4 p;
    p.c.tiles = tiles.data_ptr();
    p.c.n_pages = tiles.size(0);
    p.c.kv_heads = (int)tiles.size(1);
    p.c.page_size = (int)tiles.size(2) * 16;
    p.c.head_dim = (int)tiles.size(3) / 18;
    p.c.batch = (int)t.rows;
    p.c.page_table = static_cast<const int32_t*>(t.p);
    p.c.table_stride = t.ld;
    p.c.table_width = t.cols;
    p.c.cu_q = vec<int32_t>(a[2], at::kInt, "cu_q", t.rows + 1);
    p.c.kv_len = vec<int32_t>(a[3], at::kInt, "kv_len", t.rows);
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
        const bool bf16 = is_bf16(a[6]);
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

// what the two appends share: k, v, cos_sin, q, q_out, interleaved, dev_status from a[0] on; f makes the call
struct New {
    Heads k, v, q, o;
    Matrix cs;
    int interleaved;
    int32_t* status;
};
New fresh(PyObject* const* a, int64_t kv_heads, int64_t D) {
    New w;
    w.k = heads(a[0], "k", D);
    w.v = heads(a[1], "v", D);
    if (w.k.H != kv_heads || w.v.H != kv_heads || w.v.T != w.k.T) fail(PyExc_ValueError, "k, v", "[T, kv_heads, head_dim] each required");
    w.cs = {nullptr, 0, 0, 0};
    if (a[2] != Py_None) {
        w.cs = mat(a[2], at::kFloat, "cos_sin");
        if (w.cs.ld != w.cs.cols) fail(PyExc_ValueError, "cos_sin", "contiguous [max_pos, rot_dim] required");
    }
    w.q = w.o = {nullptr, 0, 0, 0};
    if ((a[3] == Py_None) != (a[4] == Py_None)) fail(PyExc_ValueError, "q, q_out", "both or neither required");
    if (a[3] != Py_None) {
        w.q = heads(a[3], "q", D);
        w.o = heads(a[4], "q_out", D);
        if (w.q.T != w.k.T || w.o.T != w.k.T || w.q.H != w.o.H) fail(PyExc_ValueError, "q, q_out", "one row per token each, of the same heads");
    }
    w.interleaved = PyObject_IsTrue(a[5]);
    if (w.interleaved < 0) { PyErr_Clear(); fail(PyExc_TypeError, "interleaved", "a truth value is required"); }
    w.status = status_word(a[6]);
    return w;
}

// k_cache, v_cache, page_table, cu_q, kv_len, k, v, cos_sin, q, q_out, interleaved, dev_status
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 12, [&] {
        const Paged p = paged(a);
        const New w = fresh(a + 5, p.c.kv_heads, p.c.head_dim);
        void* s = stream();
        return unlocked([&] {
            return matq_kv_append(&p.c, w.k.T, w.q.p, (int)w.q.H, w.q.ld, w.k.p, w.k.ld, w.v.p, w.v.ld, static_cast<const float*>(w.cs.p), w.cs.rows, (int)w.cs.cols,
                                  w.interleaved, w.o.p, w.o.ld, w.status, s);
        });
    });
}

// cache, page_table, cu_q, kv_len, k, v, cos_sin, q, q_out, interleaved, dev_status
PyObject* kv4_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 11, [&] {
        const Paged4 p = paged4(a);
        const New w = fresh(a + 4, p.c.kv_heads, p.c.head_dim);
        void* s = stream();
        return unlocked([&] {
            return matq_kv4_append(&p.c, w.k.T, w.q.p, (int)w.q.H, w.q.ld, w.k.p, w.k.ld, w.v.p, w.v.ld, static_cast<const float*>(w.cs.p), w.cs.rows, (int)w.cs.cols,
                                   w.interleaved, w.o.p, w.o.ld, w.status, s);
        });
    });
}

// what the two attentions share: max_q, max_kv, scale, softcap, window, out, workspace, dev_status from a[0] on
struct Attend {
    Heads q, o;
    int64_t max_q, max_kv, window;
    float scale, softcap;
    void* ws;
    size_t bytes;
    int32_t* status;
};
Attend attend(PyObject* q, PyObject* const* a, int64_t D) {
    Attend w;
    w.q = heads(q, "q", D);
    w.o = heads(a[5], "out", D);
    if (w.o.T != w.q.T || w.o.H != w.q.H) fail(PyExc_ValueError, "out", "one row per token, of q's heads");
    w.ws = nullptr;
    w.bytes = 0;
    if (a[6] != Py_None) {
        const at::Tensor& t = tensor(a[6], std::nullopt, "workspace");
        if (!t.is_contiguous()) fail(PyExc_TypeError, "workspace", "a contiguous tensor is required");
        w.ws = t.data_ptr();
        w.bytes = t.nbytes();
    }
    w.scale = (float)number(a[2], "scale");
    w.softcap = (float)number(a[3], "softcap");
    w.window = integer(a[4], "window");
    w.max_q = integer(a[0], "max_q");
    w.max_kv = integer(a[1], "max_kv");
    w.status = status_word(a[7]);
    return w;
}

// q, k_cache, v_cache, page_table, cu_q, kv_len, max_q, max_kv, scale, softcap, window, out, workspace, dev_status
PyObject* attn_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 14, [&] {
        const Paged p = paged(a + 1);
        const Attend w = attend(a[0], a + 6, p.c.head_dim);
        void* s = stream();
        return unlocked([&] {
            return matq_attn_paged(&p.c, w.q.T, w.q.p, (int)w.q.H, w.q.ld, w.scale, w.softcap, w.window, w.max_q, w.max_kv, w.o.p, w.o.ld, w.ws, w.bytes, w.status, s);
        });
    });
}

// q, cache, page_table, cu_q, kv_len, max_q, max_kv, scale, softcap, window, out, workspace, dev_status
PyObject* attn_paged4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 13, [&] {
        const Paged4 p = paged4(a + 1);
        const Attend w = attend(a[0], a + 5, p.c.head_dim);
        void* s = stream();
        return unlocked([&] {
            return matq_attn_paged4(&p.c, w.q.T, w.q.p, (int)w.q.H, w.q.ld, w.scale, w.softcap, w.window, w.max_q, w.max_kv, w.o.p, w.o.ld, w.ws, w.bytes, w.status, s);
        });
    });
}

// [N, K / group, 2] bf16, contiguous: the groups of a row
struct Groups {
    void* p;
    int64_t rows, per_row;
};
Groups groups(PyObject* o, const char* name) {
    const at::Tensor& t = tensor(o, at::kBFloat16, name);
    if (t.dim() != 3 || t.size(2) != 2 || !t.is_contiguous()) fail(PyExc_ValueError, name, "contiguous bf16 [N, K / group, 2] required");
    return {t.data_ptr(), t.size(0), t.size(1)};
}
// codes of rows without gaps
Matrix plane(PyObject* o, const char* name) {
    const Matrix m = mat(o, at::kByte, name);
    if (m.ld != m.cols) fail(PyExc_ValueError, name, "contiguous uint8 [N, K / 2] required");
    return m;
}

// W, group, packed, params, dev_status
PyObject* quantize_groups(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 5, [&] {
        const Matrix w = mat(a[0], at::kBFloat16, "W"), c = plane(a[2], "packed");
        const int group = small_integer(a[1], "group");
        const Groups g = groups(a[3], "params");
        if (c.rows != w.rows || c.cols * 2 != w.cols) fail(PyExc_ValueError, "packed", "uint8 [N, K / 2] required");
        if (group < 1 || g.rows != w.rows || g.per_row * group != w.cols) fail(PyExc_ValueError, "params", "bf16 [N, K / group, 2] required");
        int32_t* status = status_word(a[4]);
        void* s = stream();
        return unlocked([&] { return matq_quantize_groups(w.p, w.rows, w.cols, w.ld, group, static_cast<uint8_t*>(c.p), g.p, status, s); });
    });
}

// what the two linear layers share: packed, params, x, y
struct Grouped {
    Matrix c, x, y;
    Groups g;
    int group;
    int out;
};
Grouped grouped(PyObject* const* a) {
    Grouped l;
    l.c = plane(a[0], "packed");
    l.x = mat(a[2], at::kBFloat16, "x");
    l.g = groups(a[1], "params");
    if (l.x.cols != l.c.cols * 2) fail(PyExc_ValueError, "x", "packed [N, K / 2] and x [M, K] required");
    if (l.g.rows != l.c.rows || l.g.per_row < 1 || l.x.cols % l.g.per_row != 0) fail(PyExc_ValueError, "params", "bf16 [N, K / group, 2] required");
    const int64_t group = l.x.cols / l.g.per_row;
    l.group = (int)(group < 1 << 30 ? group : 0);
    const bool bf16 = is_bf16(a[3]);
    l.y = mat(a[3], bf16 ? at::kBFloat16 : at::kFloat, "y");
    if (l.y.rows != l.x.rows || l.y.cols != l.c.rows) fail(PyExc_ValueError, "y", "[M, N] required");
    l.out = bf16 ? MATQ_OUT_BF16 : MATQ_OUT_F32;
    return l;
}

// packed, params, x, y, flags
PyObject* gemv_groups(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 5, [&] {
        const Grouped l = grouped(a);
        const int flags = small_integer(a[4], "flags");
        void* s = stream();
        return unlocked([&] {
            return matq_gemv_groups(static_cast<const uint8_t*>(l.c.p), l.c.rows, l.x.cols, l.group, l.g.p, l.x.p, l.x.rows, l.x.ld, l.out, l.y.p, l.y.ld, (unsigned)flags, s);
        });
    });
}

// packed, params, x, y, workspace, dev_status
PyObject* gemm_groups(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 6, [&] {
        const Grouped l = grouped(a);
        void* ws = nullptr;
        size_t bytes = 0;
        if (a[4] != Py_None) {
            const at::Tensor& t = tensor(a[4], std::nullopt, "workspace");
            if (!t.is_contiguous()) fail(PyExc_TypeError, "workspace", "a contiguous tensor is required");
            ws = t.data_ptr();
            bytes = t.nbytes();
        }
        int32_t* status = status_word(a[5]);
        void* s = stream();
        return unlocked([&] {
            return matq_gemm_groups(static_cast<const uint8_t*>(l.c.p), l.c.rows, l.x.cols, l.group, l.g.p, l.x.p, l.x.rows, l.x.ld, l.out, l.y.p, l.y.ld, ws, bytes, status, s);
        });
    });
}

PyMethodDef methods[] = {
    {"quantize_tokens", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(quantize_tokens)), METH_FASTCALL, nullptr},
    {"gemm_a8", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gemm_a8)), METH_FASTCALL, nullptr},
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_append)), METH_FASTCALL, nullptr},
    {"attn_paged", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attn_paged)), METH_FASTCALL, nullptr},
    {"quantize_groups", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(quantize_groups)), METH_FASTCALL, nullptr},
    {"gemv_groups", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gemv_groups)), METH_FASTCALL, nullptr},
    {"gemm_groups", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gemm_groups)), METH_FASTCALL, nullptr},
    {"kv4_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv4_append)), METH_FASTCALL, nullptr},
    {"attn_paged4", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(attn_paged4)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serving", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving(void) { return PyModule_Create(&module); }

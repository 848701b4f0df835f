// Argument marshalling of the calls that a program makes per layer, in native code (Python module _qlcall): what binding.py
// checks and passes on through ctypes costs 2 to 3 us of Python per call, as long as the smallest call runs on the GPU.
//
// Each function takes the arguments of the function of binding.py that it stands for, and one to ask for the stream, and returns
// the library's status -- or None, without having called the library, for whatever is not plainly in order (an argument of another
// type, a size that does not fit, a tensor that is a view of the world of its own: subclass, batched, traced,
// without storage): binding.py then goes its own way and says what is wrong.  So every check here is one that binding.py makes as
// well, and nothing is reported from here.  One token through 1536 x 1536: 6.1 us a call through ctypes, 4.0 here.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/TensorSubclassLikeUtils.h>
#include <c10/core/impl/DeviceGuardImplInterface.h>
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstring>

#include "qlinear.h"

namespace {

struct Library {
    decltype(&ql_weight_bytes) weight_bytes;
    decltype(&ql_act_kernel_bytes) act_kernel_bytes;
    decltype(&ql_w8a8_linear) w8a8_linear;
    decltype(&ql_w4a8_linear) w4a8_linear;
    decltype(&ql_w8a8_gemm) w8a8_gemm;
    decltype(&ql_w4a8_gemm) w4a8_gemm;
    decltype(&ql_quant_act_per_token) quant_act;
    decltype(&ql_quant_act_rmsnorm) quant_rmsnorm;
    decltype(&ql_quant_act_swiglu) quant_swiglu;
    decltype(&ql_quant_act_per_token_transformed) quant_transformed;
} lib;

struct CacheLibrary {
    decltype(&ql_kv_cache_bytes) kv_cache_bytes;
    decltype(&ql_kv_resize) kv_resize;
    decltype(&ql_kv_append) kv_append;
    decltype(&ql_kv_read) kv_read;
    decltype(&ql_paged_attention) paged_attention;
} cache_lib;

PyObject *format_type = nullptr;   // binding.py's QlKvFormat

// An argument that is not in order: the caller returns None.
struct NotPlain {};
// A Python exception on its way (a keyboard interrupt may arrive wherever Python code runs): the caller passes it on.
struct Raised {};

const at::Tensor &tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) throw NotPlain();
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || at::isTensorSubclassLike(t)) throw NotPlain();
    return t;
}

const at::Tensor &tensor(PyObject *o, at::ScalarType type)
{
    const at::Tensor &t = tensor(o);
    if (t.scalar_type() != type) throw NotPlain();
    return t;
}

int as_int(int64_t v)
{
    if (v < INT_MIN || v > INT_MAX) throw NotPlain();
    return (int)v;
}

int as_int(PyObject *o)
{
    if (!PyLong_CheckExact(o)) throw NotPlain();
    int overflow = 0;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow) throw NotPlain();
    return as_int((int64_t)v);
}

float as_float(PyObject *o)
{
    if (!PyFloat_CheckExact(o)) throw NotPlain();
    return (float)PyFloat_AS_DOUBLE(o);
}

// the stream is asked for (binding.py's function) when all else is in order
void *stream_from(PyObject *ask)
{
    PyObject *o = PyObject_CallNoArgs(ask);
    if (!o) throw Raised();
    void *p = PyLong_Check(o) ? PyLong_AsVoidPtr(o) : nullptr;
    const bool failed = !PyLong_Check(o) || PyErr_Occurred();
    Py_DECREF(o);
    if (failed) throw NotPlain();   // (binding.py asks again and reports what is wrong)
    return p;
}

// any device tensor or None
template <typename T>
T *pointer(PyObject *o)
{
    return o == Py_None ? nullptr : static_cast<T *>(tensor(o).data_ptr());
}

// fp16 [rows, columns] with unit inner stride and at least one row
struct Matrix {
    void *p;
    int rows, columns;
    int64_t ld;
    explicit Matrix(PyObject *o)
    {
        const at::Tensor &t = tensor(o, at::kHalf);
        if (t.dim() != 2 || t.size(0) < 1 || t.stride(1) != 1) throw NotPlain();
        p = t.data_ptr(), rows = as_int(t.size(0)), columns = as_int(t.size(1)), ld = t.stride(0);
    }
};

struct Workspace {
    void *p = nullptr;
    size_t bytes = 0;
    explicit Workspace(PyObject *o)
    {
        if (o == Py_None) return;
        const at::Tensor &t = tensor(o);
        p = t.data_ptr(), bytes = t.nbytes();
    }
};

const void *blob(PyObject *o, int N, int K, int bits, int group)
{
    size_t need = 0;
    const at::Tensor &t = tensor(o);
    if (lib.weight_bytes(N, K, bits, group, nullptr, nullptr, &need) != QL_OK || t.nbytes() < need) throw NotPlain();
    return t.data_ptr();
}

const float *floats(PyObject *o, int64_t n)
{
    const at::Tensor &t = tensor(o, at::kFloat);
    if (t.numel() < n) throw NotPlain();
    return static_cast<const float *>(t.data_ptr());
}

const void *bias_of(PyObject *o, int N)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, at::kHalf);
    if (t.numel() < N) throw NotPlain();
    return t.data_ptr();
}

Matrix output(PyObject *o, int M, int N)
{
    const Matrix y(o);
    if (y.rows != M || y.columns != N) throw NotPlain();
    return y;
}

const int8_t *codes(PyObject *o, int M, int K)
{
    size_t need = 0;
    const at::Tensor &t = tensor(o);
    if (lib.act_kernel_bytes(M, K, &need) != QL_OK || t.nbytes() < need) throw NotPlain();
    return static_cast<const int8_t *>(t.data_ptr());
}

// The call itself, without the interpreter's lock (as ctypes makes it); None if an argument was not plain or the functions are not bound (`bound`: the address
// of one of them).
template <typename Prepare>
PyObject *call(Py_ssize_t given, Py_ssize_t wanted, bool bound, Prepare prepare)
{
    if (given != wanted || !bound) Py_RETURN_NONE;
    int status;
    try {
        auto launch = prepare();
        PyThreadState *state = PyEval_SaveThread();
        status = launch();
        PyEval_RestoreThread(state);
    } catch (const Raised &) {
        return nullptr;
    } catch (...) {   // NotPlain, or what a tensor throws when it is asked for its storage
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(status);
}

using Args = PyObject *const *;

PyObject *w8a8_linear(PyObject *, Args a, Py_ssize_t n)   // x, wq_kernel, sw, bias, N, y, ws, stream
{
    return call(n, 8, lib.weight_bytes, [&] {
        const Matrix x(a[0]);
        const int N = as_int(a[4]);
        const void *w = blob(a[1], N, x.columns, 8, 0), *b = bias_of(a[3], N);
        const float *sw = floats(a[2], N);
        const Matrix y = output(a[5], x.rows, N);
        const Workspace ws(a[6]);
        void *st = stream_from(a[7]);
        return [=] { return lib.w8a8_linear(x.p, x.ld, x.rows, x.columns, w, sw, b, N, y.p, y.ld, ws.p, ws.bytes, st); };
    });
}

PyObject *w4a8_linear(PyObject *, Args a, Py_ssize_t n)   // x, w4_kernel, group, bias, N, y, ws, stream
{
    return call(n, 8, lib.weight_bytes, [&] {
        const Matrix x(a[0]);
        const int group = as_int(a[2]), N = as_int(a[4]);
        const void *w = blob(a[1], N, x.columns, 4, group), *b = bias_of(a[3], N);
        const Matrix y = output(a[5], x.rows, N);
        const Workspace ws(a[6]);
        void *st = stream_from(a[7]);
        return [=] { return lib.w4a8_linear(x.p, x.ld, x.rows, x.columns, w, group, b, N, y.p, y.ld, ws.p, ws.bytes, st); };
    });
}

PyObject *w8a8_gemm(PyObject *, Args a, Py_ssize_t n)   // xq_kernel, sx, M, K, wq_kernel, sw, bias, N, y, ws, stream
{
    return call(n, 11, lib.weight_bytes, [&] {
        const int M = as_int(a[2]), K = as_int(a[3]), N = as_int(a[7]);
        const int8_t *xq = codes(a[0], M, K);
        const float *sx = floats(a[1], M), *sw = floats(a[5], N);
        const void *w = blob(a[4], N, K, 8, 0), *b = bias_of(a[6], N);
        const Matrix y = output(a[8], M, N);
        const Workspace ws(a[9]);
        void *st = stream_from(a[10]);
        return [=] { return lib.w8a8_gemm(xq, sx, M, K, w, sw, b, N, y.p, y.ld, ws.p, ws.bytes, st); };
    });
}

PyObject *w4a8_gemm(PyObject *, Args a, Py_ssize_t n)   // xq_kernel, sx, M, K, w4_kernel, group, bias, N, y, ws, stream
{
    return call(n, 11, lib.weight_bytes, [&] {
        const int M = as_int(a[2]), K = as_int(a[3]), group = as_int(a[5]), N = as_int(a[7]);
        const int8_t *xq = codes(a[0], M, K);
        const float *sx = floats(a[1], M);
        const void *w = blob(a[4], N, K, 4, group), *b = bias_of(a[6], N);
        const Matrix y = output(a[8], M, N);
        const Workspace ws(a[9]);
        void *st = stream_from(a[10]);
        return [=] { return lib.w4a8_gemm(xq, sx, M, K, w, group, b, N, y.p, y.ld, ws.p, ws.bytes, st); };
    });
}

PyObject *quant_act(PyObject *, Args a, Py_ssize_t n)   // x, xq_rowmajor, xq_kernel, sx, stream
{
    return call(n, 5, lib.weight_bytes, [&] {
        const Matrix x(a[0]);
        int8_t *rm = pointer<int8_t>(a[1]), *kl = pointer<int8_t>(a[2]);
        float *sx = pointer<float>(a[3]);
        void *st = stream_from(a[4]);
        return [=] { return lib.quant_act(x.p, x.ld, x.rows, x.columns, rm, kl, sx, st); };
    });
}

PyObject *quant_rmsnorm(PyObject *, Args a, Py_ssize_t n)   // x, gamma, eps, xq_rowmajor, xq_kernel, sx, stream
{
    return call(n, 7, lib.weight_bytes, [&] {
        const Matrix x(a[0]);
        const void *gamma = tensor(a[1], at::kHalf).data_ptr();
        const float eps = as_float(a[2]);
        int8_t *rm = pointer<int8_t>(a[3]), *kl = pointer<int8_t>(a[4]);
        float *sx = pointer<float>(a[5]);
        void *st = stream_from(a[6]);
        return [=] { return lib.quant_rmsnorm(x.p, x.ld, x.rows, x.columns, gamma, eps, rm, kl, sx, st); };
    });
}

PyObject *quant_swiglu(PyObject *, Args a, Py_ssize_t n)   // gate_up, xq_rowmajor, xq_kernel, sx, stream
{
    return call(n, 5, lib.weight_bytes, [&] {
        const Matrix x(a[0]);
        if (x.columns % 2) throw NotPlain();
        int8_t *rm = pointer<int8_t>(a[1]), *kl = pointer<int8_t>(a[2]);
        float *sx = pointer<float>(a[3]);
        void *st = stream_from(a[4]);
        return [=] { return lib.quant_swiglu(x.p, x.ld, x.rows, x.columns / 2, rm, kl, sx, st); };
    });
}

PyObject *quant_transformed(PyObject *, Args a, Py_ssize_t n)   // x, inv_smooth, hadamard_block, xq_rowmajor, xq_kernel, sx, stream
{
    return call(n, 7, lib.weight_bytes, [&] {
        const Matrix x(a[0]);
        const float *inv = pointer<float>(a[1]);
        const int block = as_int(a[2]);
        int8_t *rm = pointer<int8_t>(a[3]), *kl = pointer<int8_t>(a[4]);
        float *sx = pointer<float>(a[5]);
        void *st = stream_from(a[6]);
        return [=] { return lib.quant_transformed(x.p, x.ld, x.rows, x.columns, inv, block, rm, kl, sx, st); };
    });
}

// ---- the paged cache: what its calls take, checked as binding.py checks it; tensors have to be of the current device ----

struct Here {
    c10::DeviceIndex index = c10::impl::getDeviceGuardImpl(c10::DeviceType::CUDA)->getDevice().index();
    const at::Tensor &operator()(PyObject *o) const
    {
        const at::Tensor &t = tensor(o);
        if (t.get_device() != index) throw NotPlain();
        return t;
    }
    int32_t *ints(PyObject *o, int64_t n) const
    {
        const at::Tensor &t = (*this)(o);
        if (t.scalar_type() != at::kInt || t.numel() < n || !t.is_contiguous()) throw NotPlain();
        return static_cast<int32_t *>(t.data_ptr());
    }
};

struct Format {
    ql_kv_format f;
    explicit Format(PyObject *o)
    {
        if (!format_type || (PyObject *)Py_TYPE(o) != format_type) throw NotPlain();
        Py_buffer b;
        if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw NotPlain();
        const bool fits = b.len == (Py_ssize_t)sizeof(f);
        if (fits) memcpy(&f, b.buf, sizeof(f));
        PyBuffer_Release(&b);
        if (!fits || f.head_dim < 1) throw NotPlain();
    }
};

// fp16 [rows, heads * head_dim] with unit inner stride
struct Rows {
    void *p = nullptr;
    int rows = 0, heads = 0;
    int64_t ld = 0;
    Rows() {}
    Rows(const Here &here, PyObject *o, int head_dim)
    {
        const at::Tensor &t = here(o);
        if (t.scalar_type() != at::kHalf || t.dim() != 2 || t.size(0) < 1 || t.stride(1) != 1 || t.size(1) % head_dim) throw NotPlain();
        p = t.data_ptr(), rows = as_int(t.size(0)), heads = as_int(t.size(1) / head_dim);
        ld = rows > 1 ? t.stride(0) : (t.size(1) + 7) / 8 * 8;
    }
    const Rows &fit(int r, int h) const
    {
        if (rows != r || heads != h) throw NotPlain();
        return *this;
    }
};

struct Table {
    int32_t *p;
    int64_t ld;
    int columns;
    Table(const Here &here, PyObject *o, int64_t requests)
    {
        const at::Tensor &t = here(o);
        if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) < requests || t.size(0) < 1 || t.stride(1) != 1) throw NotPlain();
        p = static_cast<int32_t *>(t.data_ptr()), columns = as_int(t.size(1)), ld = t.size(0) > 1 ? t.stride(0) : t.size(1);
    }
};

void *cache_of(const Here &here, PyObject *o, const ql_kv_format &f)
{
    size_t need = 0;
    const at::Tensor &t = here(o);
    if (cache_lib.kv_cache_bytes(&f, &need) != QL_OK || !t.is_contiguous() || t.nbytes() < need) throw NotPlain();
    return t.data_ptr();
}

int as_flag(PyObject *o)
{
    if (o == Py_True) return 1;
    if (o == Py_False) return 0;
    throw NotPlain();
}

// page_size, old_len, want_len, ring, pool, pool_out, block_table, kv_len, cu_new, slots, positions, stream
PyObject *kv_resize(PyObject *, Args a, Py_ssize_t n)
{
    return call(n, 12, cache_lib.kv_cache_bytes, [&] {
        const Here here;
        const int page = as_int(a[0]), requests = as_int(here(a[1]).numel()), pages = as_int(here(a[3]).numel());
        const int most = as_int(std::min(here(a[9]).numel(), here(a[10]).numel()));
        const int32_t *old_len = here.ints(a[1], requests), *want = here.ints(a[2], requests), *pool = here.ints(a[4], 4);
        int32_t *ring = here.ints(a[3], 1), *pool_out = here.ints(a[5], 4), *kv_len = here.ints(a[7], requests);
        int32_t *cu = here.ints(a[8], (int64_t)requests + 1), *slots = here.ints(a[9], most), *positions = here.ints(a[10], most);
        const Table t(here, a[6], requests);
        void *st = stream_from(a[11]);
        return [=] {
            return cache_lib.kv_resize(old_len, want, requests, page, ring, pages, pool, pool_out, t.p, t.ld, t.columns, kv_len, cu, slots, positions, most, st);
        };
    });
}

PyObject *kv_append(PyObject *, Args a, Py_ssize_t n)   // q, k, v, cos_sin, positions, slots, q_out, cache, fmt, stream
{
    return call(n, 10, cache_lib.kv_cache_bytes, [&] {
        const Here here;
        const Format f(a[8]);
        const Rows k(here, a[1], f.f.head_dim), v(here, a[2], f.f.head_dim);
        const int T = k.rows;
        k.fit(T, f.f.heads), v.fit(T, f.f.heads);
        const float *cs = nullptr;
        const int32_t *positions = nullptr, *slots = here.ints(a[5], T);
        int rotary = 0, most = 0;
        if (a[3] != Py_None) {
            const at::Tensor &t = here(a[3]);
            if (t.scalar_type() != at::kFloat || t.dim() != 2 || !t.is_contiguous()) throw NotPlain();
            cs = static_cast<const float *>(t.data_ptr()), most = as_int(t.size(0)), rotary = as_int(t.size(1)), positions = here.ints(a[4], T);
        }
        Rows q, out;
        if (a[0] != Py_None) {
            q = Rows(here, a[0], f.f.head_dim), out = Rows(here, a[6], f.f.head_dim);
            q.fit(T, q.heads), out.fit(T, q.heads);
        } else if (a[6] != Py_None) {
            throw NotPlain();
        }
        void *cache = cache_of(here, a[7], f.f), *st = stream_from(a[9]);
        return [=] {
            return cache_lib.kv_append(q.p, q.ld, k.p, k.ld, v.p, v.ld, T, q.heads, cs, rotary, most, positions, slots, out.p, out.ld, cache, &f.f, st);
        };
    });
}

PyObject *kv_read(PyObject *, Args a, Py_ssize_t n)   // cache, fmt, slots, k, v, stream
{
    return call(n, 6, cache_lib.kv_cache_bytes, [&] {
        const Here here;
        const Format f(a[1]);
        Rows k, v;
        if (a[3] != Py_None) k = Rows(here, a[3], f.f.head_dim);
        if (a[4] != Py_None) v = Rows(here, a[4], f.f.head_dim);
        if (!k.p && !v.p) throw NotPlain();
        const int T = k.p ? k.rows : v.rows;
        if (k.p) k.fit(T, f.f.heads);
        if (v.p) v.fit(T, f.f.heads);
        const int32_t *slots = here.ints(a[2], T);
        void *cache = cache_of(here, a[0], f.f), *st = stream_from(a[5]);
        return [=] { return cache_lib.kv_read(cache, &f.f, slots, T, k.p, k.ld, v.p, v.ld, st); };
    });
}

// q, cache, fmt, block_table, cu_new, ctx_len, kv_len, scale, y, ws, causal, window, max_new, stream
PyObject *paged_attention(PyObject *, Args a, Py_ssize_t n)
{
    return call(n, 14, cache_lib.kv_cache_bytes, [&] {
        const Here here;
        const Format f(a[2]);
        const Rows q(here, a[0], f.f.head_dim), y(here, a[8], f.f.head_dim);
        y.fit(q.rows, q.heads);
        const int requests = as_int(here(a[6]).numel());
        const Table t(here, a[3], requests);
        const int32_t *cu = here.ints(a[4], (int64_t)requests + 1), *ctx = a[5] == Py_None ? nullptr : here.ints(a[5], requests), *len = here.ints(a[6], requests);
        const float scale = as_float(a[7]);
        void *ws = nullptr;
        size_t bytes = 0;
        if (a[9] != Py_None) ws = here(a[9]).data_ptr(), bytes = tensor(a[9]).nbytes();
        const int causal = as_flag(a[10]), window = as_int(a[11]), most = as_int(a[12]);
        void *cache = cache_of(here, a[1], f.f), *st = stream_from(a[13]);
        return [=] {
            return cache_lib.paged_attention(q.p, q.ld, q.rows, q.heads, cache, &f.f, t.p, t.ld, t.columns, cu, ctx, len, requests, scale, causal, window,
                                             most, y.p, y.ld, ws, bytes, st);
        };
    });
}

// bind_format(type): the class of binding.py that mirrors ql_kv_format
PyObject *bind_format(PyObject *, PyObject *type)
{
    Py_INCREF(type);
    Py_XSETREF(format_type, type);
    Py_RETURN_NONE;
}

// bind(addresses), bind_cache(addresses): the entry points of the library that binding.py has loaded, in the order of struct Library and of
// struct CacheLibrary
template <typename LIBRARY>
PyObject *bind_to(LIBRARY &to, PyObject *addresses)
{
    constexpr Py_ssize_t COUNT = sizeof(LIBRARY) / sizeof(void *);
    if (!PyTuple_CheckExact(addresses) || PyTuple_GET_SIZE(addresses) != COUNT) {
        PyErr_SetString(PyExc_TypeError, "bind takes a tuple of addresses");
        return nullptr;
    }
    void *p[COUNT];
    for (Py_ssize_t i = 0; i < COUNT; ++i) {
        p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
        if (PyErr_Occurred()) return nullptr;
    }
    static_assert(sizeof(to) == sizeof(p), "pointers only");
    memcpy(&to, p, sizeof(to));
    Py_RETURN_NONE;
}
PyObject *bind(PyObject *, PyObject *addresses) { return bind_to(lib, addresses); }
PyObject *bind_cache(PyObject *, PyObject *addresses) { return bind_to(cache_lib, addresses); }

#define QL_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {QL_METHOD(w8a8_linear), QL_METHOD(w4a8_linear), QL_METHOD(w8a8_gemm), QL_METHOD(w4a8_gemm), QL_METHOD(quant_act),
                         QL_METHOD(quant_rmsnorm), QL_METHOD(quant_swiglu), QL_METHOD(quant_transformed),
                         QL_METHOD(kv_resize), QL_METHOD(kv_append), QL_METHOD(kv_read), QL_METHOD(paged_attention),
                         {"bind", bind, METH_O, nullptr}, {"bind_cache", bind_cache, METH_O, nullptr},
                         {"bind_format", bind_format, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_qlcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__qlcall() { return PyModule_Create(&module); }

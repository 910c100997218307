// The calls of binding.py without the interpreter's share: a Python extension that reads addresses, element types and the
// current stream from torch's own objects and calls the C ABI of the library.
//
// The calls of kv_cache.py, which also have shapes and strides read, work the same way (a step's append for 16 sequences, 40 heads: 17.1 us a call
// without this, 4.4 with it; attention of one token, 2 heads, 128 keys 14.7 / 4.4).
//
// What bounds a small call is the host: on MI355X the launch itself takes 3 us and the kernel of 2 heads of 128 tokens 5.1; looking up
// torch's current stream from Python takes 2.8 us, the five tensors 0.9, the ctypes call 0.7.
// Back to back, us per call before / after: attn_fwd (1, 2, 128, 64) 8.2 / 5.2; gemm_nt (64, 64, 64) 7.4 / 3.5.
//
// Every function returns NotImplemented, having done nothing, for arguments that it does not take: then binding.py goes on
// with its own general code, which accepts, converts or refuses them.  Taken are exact tensors (no subclass, no wrapper without
// memory, no mode that wants to see the accesses) that are on the device and contiguous, or addresses as int; sizes as int in
// the range of a C int; scale as float or int; causal as bool or int; a stream as None or int; a type code as None or int.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPStream.h>

#include <climits>
#include <cstdint>
#include <type_traits>

#include "attn_fwd.h"
#include "gemm_nt.h"
#include "kv_cache.h"

namespace {

typedef decltype(&::attn_fwd) attn_fn;
typedef decltype(&::gemm_nt) gemm_fn;
static_assert(std::is_same<attn_fn, decltype(&::attn_fwd_fp8)>::value && std::is_same<gemm_fn, decltype(&::gemm_nt_fp8)>::value, "pairs of calls");

attn_fn attn_calls[2];          // attn_fwd, attn_fwd_fp8
gemm_fn gemm_calls[2];          // gemm_nt, gemm_nt_fp8
bool enabled = false;

PyObject* not_taken()
{
    Py_RETURN_NOTIMPLEMENTED;
}

// Address of a tensor (or an int), and the tensor itself where it is one.
bool address(PyObject* x, void*& p, const at::Tensor*& t)
{
    t = nullptr;
    if (THPVariable_CheckExact(x)) {
        const at::Tensor& a = THPVariable_Unpack(x);
        const c10::DispatchKeySet keys = a.key_set();
        if (!a.defined() || !a.is_cuda() || a.layout() != at::kStrided || !a.has_storage() || keys.has(c10::DispatchKey::Functionalize) ||
            keys.has(c10::DispatchKey::Python) || keys.has(c10::DispatchKey::FuncTorchGradWrapper) ||
            keys.has(c10::DispatchKey::FuncTorchBatched) || !a.is_contiguous())
            return false;
        p = a.data_ptr();
        t = &a;
        return true;
    }
    if (!PyLong_CheckExact(x)) return false;
    p = reinterpret_cast<void*>(PyLong_AsUnsignedLongLong(x));
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

bool c_int(PyObject* x, int& v)
{
    if (!PyLong_CheckExact(x)) return false;
    int overflow = 0;
    const long long l = PyLong_AsLongLongAndOverflow(x, &overflow);
    if (overflow || l < INT_MIN || l > INT_MAX) return false;
    v = (int)l;
    return true;
}

// The stream to launch on: the one given, or torch's current one (some tensor is on the device, so torch has initialised it).
bool stream_of(PyObject* x, bool have_tensor, void*& s)
{
    if (x == Py_None) {
        if (!have_tensor) return false;
        s = c10::hip::getCurrentHIPStream().stream();
        return true;
    }
    if (!PyLong_CheckExact(x)) return false;
    s = reinterpret_cast<void*>(PyLong_AsUnsignedLongLong(x));
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

// The type code given, or that of the tensor's 16-bit elements.
bool code_of(PyObject* x, const at::Tensor* t, int& code)
{
    if (x != Py_None) return c_int(x, code);
    if (!t) return false;
    if (t->scalar_type() == at::kHalf) code = 0;
    else if (t->scalar_type() == at::kBFloat16) code = 1;
    else return false;
    return true;
}

// (q, k, v, o, lse, B, H, N, d, scale, causal, stream, type code)
template <int WHICH>            // 0: 16-bit inputs, whose type is the code; 1: E4M3 inputs, the code is the type of o
PyObject* attn(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != 13 || !enabled || at::impl::torch_function_mode_enabled()) return not_taken();
    try {
        void* p[5];
        const at::Tensor* t[5];
        bool tensors = false;
        for (int i = 0; i < 5; ++i) {
            if (!address(args[i], p[i], t[i])) return not_taken();
            tensors |= t[i] != nullptr;
        }
        int size[4], code;
        for (int i = 0; i < 4; ++i)
            if (!c_int(args[5 + i], size[i])) return not_taken();
        if (!PyFloat_CheckExact(args[9]) && !PyLong_CheckExact(args[9])) return not_taken();
        const double scale = PyFloat_AsDouble(args[9]);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return not_taken();
        }
        if (!PyBool_Check(args[10]) && !PyLong_CheckExact(args[10])) return not_taken();
        const int causal = PyObject_IsTrue(args[10]);
        void* stream;
        if (!stream_of(args[11], tensors, stream) || !code_of(args[12], t[WHICH == 0 ? 0 : 3], code)) return not_taken();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = attn_calls[WHICH](p[0], p[1], p[2], p[3], (float*)p[4], size[0], size[1], size[2], size[3], (float)scale, causal, stream, code);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (...) {             // (torch's: the general code meets the same and reports it)
        return not_taken();
    }
}

// (a, b, c, M, N, K, stream, type code)
template <int WHICH>
PyObject* gemm(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != 8 || !enabled || at::impl::torch_function_mode_enabled()) return not_taken();
    try {
        void* p[3];
        const at::Tensor* t[3];
        bool tensors = false;
        for (int i = 0; i < 3; ++i) {
            if (!address(args[i], p[i], t[i])) return not_taken();
            tensors |= t[i] != nullptr;
        }
        int size[3], code;
        for (int i = 0; i < 3; ++i)
            if (!c_int(args[3 + i], size[i])) return not_taken();
        void* stream;
        if (!stream_of(args[6], tensors, stream) || !code_of(args[7], WHICH == 0 ? t[0] : nullptr, code)) return not_taken();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = gemm_calls[WHICH](p[0], p[1], p[2], size[0], size[1], size[2], stream, code);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (...) {
        return not_taken();
    }
}

// ---- the operators around the paged cache

struct KvCalls {
    decltype(&::attn_paged) attn_paged;
    decltype(&::kv_append) kv_append;
    decltype(&::rope) rope;
    decltype(&::kv_reserve) kv_reserve;
    decltype(&::kv_free) kv_free;
    decltype(&::kv_fork) kv_fork;
    decltype(&::kv_compact) kv_compact;
    decltype(&::kv_copy_pages) kv_copy_pages;
} kv_calls;
bool kv_enabled = false;

// What is wrong with a call's arguments is for the general code to say: it is given up here by this.
struct NotTaken {};
void want(bool ok) { if (!ok) throw NotTaken(); }

// The tensors of a call: exact ones on the current device.
class Args {
    PyObject* const* args_;
    int device_;

public:
    Args(PyObject* const* args) : args_(args), device_(-1) {}
    bool none(int i) const { return args_[i] == Py_None; }
    const at::Tensor& tensor(int i)
    {
        want(THPVariable_CheckExact(args_[i]));
        const at::Tensor& a = THPVariable_Unpack(args_[i]);
        const c10::DispatchKeySet keys = a.key_set();
        want(a.defined() && a.is_cuda() && a.layout() == at::kStrided && a.has_storage() && !keys.has(c10::DispatchKey::Functionalize) &&
             !keys.has(c10::DispatchKey::Python) && !keys.has(c10::DispatchKey::FuncTorchGradWrapper) && !keys.has(c10::DispatchKey::FuncTorchBatched));
        if (device_ < 0) device_ = c10::hip::current_device();
        want(a.device().index() == device_);
        return a;
    }
    // A contiguous array of a type, of n elements unless n < 0.
    void* array(int i, at::ScalarType type, int64_t n, int64_t* found = nullptr)
    {
        const at::Tensor& a = tensor(i);
        want(a.scalar_type() == type && a.is_contiguous() && (n < 0 || a.numel() == n));
        if (found) *found = a.numel();
        return a.data_ptr();
    }
    int whole(int i) const
    {
        int v;
        want(c_int(args_[i], v));
        return v;
    }
    bool truth(int i) const
    {
        want(PyBool_Check(args_[i]) || PyLong_CheckExact(args_[i]));
        return PyObject_IsTrue(args_[i]) != 0;
    }
    float real(int i) const
    {
        want(PyFloat_CheckExact(args_[i]) || PyLong_CheckExact(args_[i]));
        const double x = PyFloat_AsDouble(args_[i]);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            throw NotTaken();
        }
        return (float)x;
    }
    void* stream(int i) const
    {
        void* s;
        want(stream_of(args_[i], true, s));
        return s;
    }
};

int narrow(int64_t x)
{
    want(x >= INT_MIN && x <= INT_MAX);
    return (int)x;
}
int type_of(const at::Tensor& t)
{
    switch (t.scalar_type()) {
        case at::kHalf: return KV_FP16;
        case at::kBFloat16: return KV_BF16;
        case at::kFloat8_e4m3fn: case at::kByte: return KV_E4M3;
        default: throw NotTaken();
    }
}
// [layers,] pages, heads, page size, d of both, scales of the heads
kv_pages pages_of(Args& a, int k, int v, int k_scale, int v_scale, bool layers)
{
    const at::Tensor &x = a.tensor(k), &y = a.tensor(v);
    const int first = layers ? 1 : 0;
    want(x.dim() == 4 + first && x.sizes() == y.sizes() && x.strides() == y.strides() && x.scalar_type() == y.scalar_type());
    want(x.stride(3 + first) == 1);
    kv_pages p{};
    p.k = x.data_ptr();
    p.v = y.data_ptr();
    p.layer_stride = layers ? x.stride(0) : 0;
    p.page_stride = x.stride(first);
    p.head_stride = x.stride(first + 1);
    p.token_stride = x.stride(first + 2);
    p.layers = layers ? narrow(x.size(0)) : 1;
    p.pages = narrow(x.size(first));
    p.heads = narrow(x.size(first + 1));
    p.page_size = narrow(x.size(first + 2));
    p.d = narrow(x.size(first + 3));
    p.dtype = type_of(x);
    if (k_scale >= 0 && !a.none(k_scale)) p.k_scale = (const float*)a.array(k_scale, at::kFloat, p.heads);
    if (v_scale >= 0 && !a.none(v_scale)) p.v_scale = (const float*)a.array(v_scale, at::kFloat, p.heads);
    return p;
}
// q_start, kv_len, table are arguments i, i + 1, i + 2
kv_batch batch_of(Args& a, int i, int64_t tokens, int max_q, int max_kv)
{
    kv_batch b{};
    int64_t n;
    b.kv_len = (const int*)a.array(i + 1, at::kInt, -1, &n);
    b.q_start = (const int*)a.array(i, at::kInt, n + 1);
    const at::Tensor& t = a.tensor(i + 2);
    want(a.tensor(i + 1).dim() == 1 && t.scalar_type() == at::kInt && t.dim() == 2 && t.size(0) == n && t.stride(1) == 1);
    b.table = (const int*)t.data_ptr();
    b.sequences = narrow(n);
    b.tokens = narrow(tokens);
    b.table_width = narrow(t.size(1));
    b.table_stride = narrow(t.stride(0));
    b.max_q = max_q;
    b.max_kv = max_kv;
    return b;
}
kv_rows rows_of(const at::Tensor& t, int64_t tokens, int64_t heads, int64_t d, at::ScalarType type)
{
    want(t.dim() == 3 && t.size(0) == tokens && t.size(1) == heads && t.size(2) == d && t.stride(2) == 1 && t.scalar_type() == type);
    return {t.data_ptr(), t.stride(0), t.stride(1)};
}
// ref, table, kv_len are arguments i, i + 1, i + 2
kv_book book_of(Args& a, int i, int page_size)
{
    kv_book b{};
    int64_t pages, rows;
    b.ref = (int*)a.array(i, at::kInt, -1, &pages);
    b.kv_len = (int*)a.array(i + 2, at::kInt, -1, &rows);
    const at::Tensor& t = a.tensor(i + 1);
    want(a.tensor(i + 2).dim() == 1 && t.scalar_type() == at::kInt && t.dim() == 2 && t.size(0) == rows && t.stride(1) == 1);
    b.table = (int*)t.data_ptr();
    b.pages = narrow(pages);
    b.rows = narrow(rows);
    b.table_width = narrow(t.size(1));
    b.table_stride = narrow(t.stride(0));
    b.page_size = page_size;
    return b;
}

template <int COUNT, typename Call> PyObject* kv_call(PyObject* const* args, Py_ssize_t n, Call call)
{
    if (n != COUNT || !enabled || !kv_enabled || at::impl::torch_function_mode_enabled()) return not_taken();
    try {
        Args a(args);
        return PyLong_FromLong(call(a));
    } catch (...) {             // (NotTaken, and torch's: the general code meets the same and reports it)
        return not_taken();
    }
}
template <typename Call> int unlocked(Call call)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}

// (q, k_cache, v_cache, q_start, kv_len, table, o, lse, max_q, max_kv, scale, causal, k_scale, v_scale, workspace, stream)
PyObject* attn_paged_(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return kv_call<16>(args, n, [](Args& a) {
        const at::Tensor& q = a.tensor(0);
        want(q.dim() == 3);
        const kv_rows rq = rows_of(q, q.size(0), q.size(1), q.size(2), q.scalar_type()), ro = rows_of(a.tensor(6), q.size(0), q.size(1), q.size(2), q.scalar_type());
        const kv_pages c = pages_of(a, 1, 2, 12, 13, false);
        want(c.d == q.size(2));
        const kv_batch b = batch_of(a, 3, q.size(0), a.whole(8), a.whole(9));
        float* lse = nullptr;
        if (!a.none(7)) {
            lse = (float*)a.array(7, at::kFloat, q.size(0) * q.size(1));
            want(a.tensor(7).dim() == 2 && a.tensor(7).size(0) == q.size(0));
        }
        int64_t bytes = 0;
        void* const ws = a.none(14) ? nullptr : a.array(14, at::kByte, -1, &bytes);
        const int heads = narrow(q.size(1)), causal = a.truth(11), type = type_of(q);
        const float scale = a.real(10);
        void* const stream = a.stream(15);
        return unlocked([&] { return kv_calls.attn_paged(&c, &b, &rq, &ro, lse, heads, scale, causal, type, ws, bytes, stream); });
    });
}

// (k, v, k_cache, v_cache, q_start, kv_len, table, max_q, max_kv, q, q_out, freq, layout, amplitude, k_scale, v_scale, stream)
PyObject* kv_append_(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return kv_call<17>(args, n, [](Args& a) {
        const at::Tensor& k = a.tensor(0);
        want(k.dim() == 3);
        const at::ScalarType type = k.scalar_type();
        const kv_pages c = pages_of(a, 2, 3, 14, 15, false);
        const kv_rows rk = rows_of(k, k.size(0), c.heads, c.d, type), rv = rows_of(a.tensor(1), k.size(0), c.heads, c.d, type);
        const kv_batch b = batch_of(a, 4, k.size(0), a.whole(7), a.whole(8));
        kv_rows rq{}, ro{};
        int heads = 0;
        if (!a.none(9)) {
            const at::Tensor& q = a.tensor(9);
            want(q.dim() == 3);
            heads = narrow(q.size(1));
            rq = rows_of(q, k.size(0), heads, c.d, type);
            ro = rows_of(a.tensor(10), k.size(0), heads, c.d, type);
        } else {
            want(a.none(10));
        }
        int64_t half = 0;
        const double* const freq = a.none(11) ? nullptr : (const double*)a.array(11, at::kDouble, -1, &half);
        const int layout = a.whole(12), code = type_of(k), rot = narrow(2 * half);
        const float amplitude = a.real(13);
        void* const stream = a.stream(16);
        return unlocked([&] { return kv_calls.kv_append(&c, &b, &rk, &rv, &rq, &ro, heads, freq, rot, layout, amplitude, code, stream); });
    });
}

// (x, y, freq, pos, layout, amplitude, inverse, stream)
PyObject* rope_(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return kv_call<8>(args, n, [](Args& a) {
        const at::Tensor &x = a.tensor(0), &y = a.tensor(1);
        want(x.dim() == 4 && x.sizes() == y.sizes() && x.scalar_type() == y.scalar_type() && x.stride(3) == 1 && y.stride(3) == 1);
        const rope_tensor tx{x.data_ptr(), x.stride(0), x.stride(1), x.stride(2)}, ty{y.data_ptr(), y.stride(0), y.stride(1), y.stride(2)};
        int64_t half, stride = 0;
        const double* const freq = (const double*)a.array(2, at::kDouble, -1, &half);
        const int* pos = nullptr;
        if (!a.none(3)) {
            const at::Tensor& p = a.tensor(3);
            want((p.dim() == 1 && p.size(0) == x.size(2)) || (p.dim() == 2 && p.size(0) == x.size(0) && p.size(1) == x.size(2)));
            pos = (const int*)a.array(3, at::kInt, -1);
            stride = p.dim() == 2 ? x.size(2) : 0;
        }
        const int b = narrow(x.size(0)), h = narrow(x.size(1)), t = narrow(x.size(2)), d = narrow(x.size(3)), layout = a.whole(4), inverse = a.truth(6), code = type_of(x);
        const int rot = narrow(2 * half);
        const float amplitude = a.real(5);
        void* const stream = a.stream(7);
        return unlocked([&] { return kv_calls.rope(&tx, &ty, b, h, t, d, pos, stride, freq, rot, layout, amplitude, inverse, code, stream); });
    });
}

// (ref, table, kv_len, rows, new_len, missing, page_size, stream)
PyObject* kv_reserve_(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return kv_call<8>(args, n, [](Args& a) {
        const kv_book b = book_of(a, 0, a.whole(6));
        int64_t count;
        const int* const list = (const int*)a.array(3, at::kInt, -1, &count);
        const int* const len = (const int*)a.array(4, at::kInt, count);
        int* const missing = (int*)a.array(5, at::kInt, 1);
        want(a.tensor(3).dim() == 1 && a.tensor(4).dim() == 1 && count <= KV_MAX_LIST);
        void* const stream = a.stream(7);
        return unlocked([&] { return kv_calls.kv_reserve(&b, list, len, (int)count, missing, stream); });
    });
}

// (ref, table, kv_len, rows, page_size, stream)
PyObject* kv_free_(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return kv_call<6>(args, n, [](Args& a) {
        const kv_book b = book_of(a, 0, a.whole(4));
        int64_t count;
        const int* const list = (const int*)a.array(3, at::kInt, -1, &count);
        want(a.tensor(3).dim() == 1 && count <= KV_MAX_LIST);
        void* const stream = a.stream(5);
        return unlocked([&] { return kv_calls.kv_free(&b, list, (int)count, stream); });
    });
}

// (k_cache, v_cache, ref, table, kv_len, src, dst, missing, stream)
PyObject* kv_fork_(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return kv_call<9>(args, n, [](Args& a) {
        const kv_pages c = pages_of(a, 0, 1, -1, -1, true);
        const kv_book b = book_of(a, 2, c.page_size);
        int64_t count;
        const int* const src = (const int*)a.array(5, at::kInt, -1, &count);
        const int* const dst = (const int*)a.array(6, at::kInt, count);
        int* const missing = (int*)a.array(7, at::kInt, 1);
        want(a.tensor(5).dim() == 1 && a.tensor(6).dim() == 1 && count <= KV_MAX_LIST);
        void* const stream = a.stream(8);
        return unlocked([&] { return kv_calls.kv_fork(&c, &b, src, dst, (int)count, missing, stream); });
    });
}

// (k_cache, v_cache, ref, table, kv_len, workspace, stream)
PyObject* kv_compact_(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return kv_call<7>(args, n, [](Args& a) {
        const kv_pages c = pages_of(a, 0, 1, -1, -1, true);
        const kv_book b = book_of(a, 2, c.page_size);
        int64_t bytes;
        void* const workspace = a.array(5, at::kByte, -1, &bytes);
        void* const stream = a.stream(6);
        return unlocked([&] { return kv_calls.kv_compact(&c, &b, workspace, bytes, stream); });
    });
}

// (k_cache, v_cache, src, dst, stream)
PyObject* kv_copy_pages_(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return kv_call<5>(args, n, [](Args& a) {
        const kv_pages c = pages_of(a, 0, 1, -1, -1, true);
        int64_t count;
        const int* const src = (const int*)a.array(2, at::kInt, -1, &count);
        const int* const dst = (const int*)a.array(3, at::kInt, count);
        want(a.tensor(2).dim() == 1 && a.tensor(3).dim() == 1 && count <= KV_MAX_LIST);
        void* const stream = a.stream(4);
        return unlocked([&] { return kv_calls.kv_copy_pages(&c, src, dst, (int)count, stream); });
    });
}

// bind_kv(attn_paged, kv_append, rope, kv_reserve, kv_free, kv_fork, kv_compact, kv_copy_pages): addresses of the functions of the loaded library
PyObject* bind_kv(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    void* f[8];
    if (n != 8) {
        PyErr_SetString(PyExc_TypeError, "bind_kv takes eight addresses");
        return nullptr;
    }
    for (int i = 0; i < 8; ++i) {
        f[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
        if (!f[i]) {
            PyErr_SetString(PyExc_ValueError, "bind_kv takes eight addresses");
            return nullptr;
        }
    }
    kv_calls = {(decltype(&::attn_paged))f[0], (decltype(&::kv_append))f[1], (decltype(&::rope))f[2],
                (decltype(&::kv_reserve))f[3], (decltype(&::kv_free))f[4], (decltype(&::kv_fork))f[5],
                (decltype(&::kv_compact))f[6], (decltype(&::kv_copy_pages))f[7]};
    kv_enabled = true;
    Py_RETURN_NONE;
}

// bind(attn_fwd, attn_fwd_fp8, gemm_nt, gemm_nt_fp8): addresses of the functions of the loaded library
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    void* f[4];
    if (n != 4) {
        PyErr_SetString(PyExc_TypeError, "bind takes four addresses");
        return nullptr;
    }
    for (int i = 0; i < 4; ++i) {
        f[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
        if (!f[i]) {
            PyErr_SetString(PyExc_ValueError, "bind takes four addresses");
            return nullptr;
        }
    }
    attn_calls[0] = (attn_fn)f[0];
    attn_calls[1] = (attn_fn)f[1];
    gemm_calls[0] = (gemm_fn)f[2];
    gemm_calls[1] = (gemm_fn)f[3];
    enabled = true;
    Py_RETURN_NONE;
}

// disable(): from here on nothing is taken (a forked child: torch refuses its device there, in the general code)
PyObject* disable(PyObject*, PyObject*)
{
    enabled = false;
    Py_RETURN_NONE;
}

template <typename F> PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"attn_fwd", fast(attn<0>), METH_FASTCALL, nullptr},
    {"attn_fwd_fp8", fast(attn<1>), METH_FASTCALL, nullptr},
    {"gemm_nt", fast(gemm<0>), METH_FASTCALL, nullptr},
    {"gemm_nt_fp8", fast(gemm<1>), METH_FASTCALL, nullptr},
    {"attn_paged", fast(attn_paged_), METH_FASTCALL, nullptr},
    {"kv_append", fast(kv_append_), METH_FASTCALL, nullptr},
    {"rope", fast(rope_), METH_FASTCALL, nullptr},
    {"kv_reserve", fast(kv_reserve_), METH_FASTCALL, nullptr},
    {"kv_free", fast(kv_free_), METH_FASTCALL, nullptr},
    {"kv_fork", fast(kv_fork_), METH_FASTCALL, nullptr},
    {"kv_compact", fast(kv_compact_), METH_FASTCALL, nullptr},
    {"kv_copy_pages", fast(kv_copy_pages_), METH_FASTCALL, nullptr},
    {"bind", fast(bind), METH_FASTCALL, nullptr},
    {"bind_kv", fast(bind_kv), METH_FASTCALL, nullptr},
    {"disable", disable, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch that the extension was compiled against, whose object layouts it knows (binding.py compares).
PyMODINIT_FUNC PyInit__fastcall(void)
{
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", FASTCALL_TORCH) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}

// Argument marshalling of the attention's tensor calls in native code (Python extension module _attention_marshal), as
// torch_marshal.cpp does it for the output layer: a decoding step's calls are bound by the host.  These functions take the calls that a
// program makes all the time -- plain tensors on the current device and stream, all arguments valid -- and return None for every
// other call, which attention.py then takes through its own code: the checks and their messages stand there, once.
//
//   None            not a call for this path
//   int             the library's non-zero status
//   tensor, tuple   the outputs, as attention.py returns them
//
// Nothing is kept between calls but the addresses of the library's entry points and the function that names the current stream.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty_cuda_dispatch.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/wht_attention.h"

namespace {

decltype(&wht_attention_append) lib_append;
decltype(&wht_attention_workspace_bytes) lib_workspace_bytes;
decltype(&wht_attention_paged) lib_paged;
PyObject* raw_stream_of;                // torch._C._cuda_getCurrentRawStream

bool modes_active() {
    return at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set();
}

PyObject* none() { Py_RETURN_NONE; }

// The tensors of one call.  `ok` turns false where this path does not take one.
struct Call {
    c10::Device device{c10::DeviceType::CUDA, 0};
    at::ScalarType type = at::kFloat;
    int64_t pages = 0, heads = 0, page_size = 0, head_dim = 0;
    wht_attention_cache_t cache{};
    wht_attention_batch_t batch{};
    bool ok = true;

    // A tensor on the GPU with memory of its own and nothing wrapped around it.
    const at::Tensor* plain(PyObject* obj) {
        static const c10::DispatchKeySet ordinary({c10::DispatchKey::CUDA, c10::DispatchKey::ADInplaceOrView,
                                                   c10::DispatchKey::AutogradCUDA, c10::DispatchKey::AutocastCUDA});
        if (!THPVariable_CheckExact(obj)) return refuse();
        const at::Tensor& t = THPVariable_Unpack(obj);
        if (!t.defined() || (t.key_set() | ordinary) != ordinary || !t.is_cuda()) return refuse();
        return &t;
    }
    const at::Tensor* refuse() { ok = false; return nullptr; }

    void take_cache(PyObject* k_obj, PyObject* v_obj) {
        if (modes_active()) { ok = false; return; }
        const at::Tensor *k = plain(k_obj), *v = plain(v_obj);
        if (!ok || k->dim() != 4 || v->dim() != 4 || k->sizes() != v->sizes() || k->strides() != v->strides() || k->scalar_type() != v->scalar_type() ||
            k->device() != v->device() || k->stride(3) != 1) { ok = false; return; }
        type = k->scalar_type();
        device = k->device();
        const c10::impl::VirtualGuardImpl guard(c10::DeviceType::CUDA);
        if ((type != at::kFloat && type != at::kBFloat16) || guard.getDevice() != device) { ok = false; return; }
        pages = k->size(0); heads = k->size(1); page_size = k->size(2); head_dim = k->size(3);
        if (k->numel() == 0 || pages > INT32_MAX || heads > INT32_MAX || page_size > INT32_MAX) { ok = false; return; }
        cache = {k->data_ptr(), v->data_ptr(), k->stride(0), k->stride(1), k->stride(2), (int32_t)pages, (int32_t)heads, (int32_t)page_size, (int32_t)head_dim};
    }
    // int32 [n], or [n][width]
    const int32_t* ints(PyObject* obj, int64_t dims, int64_t n) {
        const at::Tensor* t = plain(obj);
        if (!t || t->dim() != dims || t->scalar_type() != at::kInt || t->device() != device || (n >= 0 && t->size(0) != n) ||
            (t->size(dims - 1) > 1 && t->stride(dims - 1) != 1)) { ok = false; return nullptr; }
        return static_cast<const int32_t*>(t->data_ptr());
    }
    void take_batch(PyObject* table, PyObject* lengths, PyObject* starts, int64_t T) {
        batch.table = ints(table, 2, -1);
        if (!ok) return;
        const at::Tensor& t = THPVariable_Unpack(table);
        const int64_t B = t.size(0), width = t.size(1);
        if (B == 0 || B > INT32_MAX || width > INT32_MAX) { ok = false; return; }
        batch.lengths = ints(lengths, 1, B);
        if (starts != Py_None) batch.q_starts = ints(starts, 1, B + 1);
        else if (T != B) ok = false;
        batch.table_stride = t.stride(0);
        batch.B = (int32_t)B;
        batch.width = (int32_t)width;
    }
    // [T][heads][head_dim]; n < 0: any number of heads
    const at::Tensor* rows(PyObject* obj, wht_attention_rows_t& r, int64_t T, int64_t n) {
        const at::Tensor* t = plain(obj);
        if (!t || t->dim() != 3 || t->size(2) != head_dim || t->stride(2) != 1 || t->scalar_type() != type || t->device() != device ||
            (T >= 0 && t->size(0) != T) || (n >= 0 && t->size(1) != n) || t->size(0) == 0 || t->size(1) > INT32_MAX) return refuse();
        r = {t->data_ptr(), t->stride(0), t->stride(1)};
        return t;
    }
    int32_t dtype() const { return type == at::kFloat ? WHT_DTYPE_F32 : WHT_DTYPE_BF16; }
    at::Tensor empty(c10::IntArrayRef sizes, at::ScalarType t) const { return at::cuda::empty(sizes, at::TensorOptions().device(device).dtype(t)); }
    bool stream(void** to) const {
        PyObject* index = PyLong_FromLong(device.index());
        if (!index) return false;
        PyObject* handle = PyObject_CallOneArg(raw_stream_of, index);
        Py_DECREF(index);
        if (!handle) return false;
        *to = PyLong_AsVoidPtr(handle);
        Py_DECREF(handle);
        return !PyErr_Occurred();
    }
};

// A Python int in [least, most]; `ok` is false for anything else.
int64_t whole(PyObject* obj, int64_t least, int64_t most, bool& ok) {
    if (!PyLong_CheckExact(obj)) { ok = false; return 0; }
    int over = 0;
    const int64_t x = PyLong_AsLongLongAndOverflow(obj, &over);
    if (over || x < least || x > most) ok = false;
    return x;
}

bool expect(Py_ssize_t got, Py_ssize_t want) {
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
    return false;
}

// append(q | None, k, v, k_pages, v_pages, table, lengths, rope | None, q_starts | None, position, interleaved, q_out | None)
PyObject* append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!expect(nargs, 12)) return nullptr;
    Call c;
    c.take_cache(args[3], args[4]);
    if (!c.ok) return none();
    wht_attention_rows_t q{}, k{}, v{}, out{};
    const at::Tensor* kt = c.rows(args[1], k, -1, c.heads);
    if (!c.ok) return none();
    const int64_t T = kt->size(0);
    c.rows(args[2], v, T, c.heads);
    const at::Tensor* qt = args[0] == Py_None ? nullptr : c.rows(args[0], q, T, -1);
    c.take_batch(args[5], args[6], args[8], T);
    const int64_t position = whole(args[9], 0, INT64_MAX, c.ok);
    const int interleaved = PyObject_IsTrue(args[10]);
    if (interleaved < 0) return nullptr;
    const float* rope = nullptr;
    int64_t rope_rows = 0, rotary = 0;
    if (c.ok && args[7] != Py_None) {
        const at::Tensor* r = c.plain(args[7]);
        if (!r || r->scalar_type() != at::kFloat || r->dim() != 3 || r->size(2) != 2 || !r->is_contiguous() || r->device() != c.device || r->numel() == 0 ||
            r->size(1) > INT32_MAX / 2) return none();
        rope = static_cast<const float*>(r->data_ptr());
        rope_rows = r->size(0);
        rotary = 2 * r->size(1);
    }
    if (qt && args[11] != Py_None) c.rows(args[11], out, T, qt->size(1));
    if (!c.ok) return none();
    PyObject* result = nullptr;                                     // owned
    if (!qt) result = Py_NewRef(Py_None);
    else if (args[11] != Py_None) result = Py_NewRef(args[11]);
    else {
        at::Tensor t = c.empty(qt->sizes(), c.type);
        out = {t.data_ptr(), t.stride(0), t.stride(1)};
        result = THPVariable_Wrap(std::move(t));
    }
    void* stream = nullptr;
    if (!result || !c.stream(&stream)) { Py_XDECREF(result); return nullptr; }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = lib_append(&q, &k, &v, &out, T, qt ? (int32_t)qt->size(1) : 0, &c.cache, &c.batch, rope, rope_rows, (int32_t)rotary, interleaved, position,
                    c.dtype(), stream);
    Py_END_ALLOW_THREADS
    if (rc != WHT_OK) { Py_DECREF(result); return PyLong_FromLong(rc); }
    // None would say that the call was declined
    if (!qt) { Py_DECREF(result); return PyTuple_New(0); }
    return result;
    END_HANDLE_TH_ERRORS
}

// paged(q, k_pages, v_pages, table, lengths, q_starts | None, prefix_table | None, prefix_length, max_q | None, max_length | None, scale | None,
//       out | None, lse | None, want_lse, workspace | None)
PyObject* paged(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!expect(nargs, 15)) return nullptr;
    Call c;
    c.take_cache(args[1], args[2]);
    if (!c.ok) return none();
    wht_attention_rows_t q{}, o{};
    const at::Tensor* qt = c.rows(args[0], q, -1, -1);
    if (!c.ok) return none();
    const int64_t T = qt->size(0), q_heads = qt->size(1);
    c.take_batch(args[3], args[4], args[5], T);
    const int want_lse = PyObject_IsTrue(args[13]);
    if (want_lse < 0) return nullptr;
    const int64_t prefix = whole(args[7], 0, (int64_t)1 << 30, c.ok);
    const int32_t* prefix_table = nullptr;
    if (c.ok && prefix > 0) {
        if (args[6] == Py_None) return none();
        prefix_table = c.ints(args[6], 1, -1);
        if (!c.ok || THPVariable_Unpack(args[6]).size(0) < (prefix + c.page_size - 1) / c.page_size) return none();
    }
    const int64_t max_q = args[8] != Py_None ? whole(args[8], 1, INT32_MAX, c.ok) : c.batch.q_starts ? T : 1;
    const int64_t max_length = args[9] != Py_None ? whole(args[9], 0, INT64_MAX, c.ok) : (int64_t)c.batch.width * c.page_size;
    double scale = 1.0 / std::sqrt((double)c.head_dim);
    if (args[10] != Py_None) {
        if (!PyFloat_CheckExact(args[10])) return none();
        scale = PyFloat_AS_DOUBLE(args[10]);
    }
    if (c.ok && args[11] != Py_None) c.rows(args[11], o, T, q_heads);
    float* lse = nullptr;
    if (c.ok && args[12] != Py_None) {
        const at::Tensor* t = c.plain(args[12]);
        if (!t || t->scalar_type() != at::kFloat || t->dim() != 2 || t->size(0) != T || t->size(1) != q_heads || !t->is_contiguous() || t->device() != c.device)
            return none();
        lse = static_cast<float*>(t->data_ptr());
    }
    if (!c.ok) return none();
    const size_t need = lib_workspace_bytes(T, c.batch.B, (int32_t)q_heads, (int32_t)c.heads, (int32_t)c.head_dim, (int32_t)max_q, max_length, prefix, c.dtype());
    void* ws = nullptr;
    size_t ws_bytes = 0;
    at::Tensor made_ws;
    if (args[14] != Py_None) {
        const at::Tensor* t = c.plain(args[14]);
        if (!t || !t->is_contiguous() || t->device() != c.device) return none();
        ws = t->data_ptr();
        ws_bytes = t->nbytes();
    } else if (need > 0) {
        made_ws = c.empty({(int64_t)need}, at::kByte);
        ws = made_ws.data_ptr();
        ws_bytes = need;
    }
    at::Tensor made_out, made_lse;
    if (args[11] == Py_None) {
        made_out = c.empty(qt->sizes(), c.type);
        o = {made_out.data_ptr(), made_out.stride(0), made_out.stride(1)};
    }
    if (!lse && want_lse) {
        made_lse = c.empty({T, q_heads}, at::kFloat);
        lse = static_cast<float*>(made_lse.data_ptr());
    }
    PyObject* out = made_out.defined() ? THPVariable_Wrap(std::move(made_out)) : Py_NewRef(args[11]);       // owned, both
    PyObject* out_lse = !lse ? nullptr : made_lse.defined() ? THPVariable_Wrap(std::move(made_lse)) : Py_NewRef(args[12]);
    void* stream = nullptr;
    if (!out || (lse && !out_lse) || !c.stream(&stream)) { Py_XDECREF(out); Py_XDECREF(out_lse); return nullptr; }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = lib_paged(&q, &o, lse, T, (int32_t)q_heads, &c.cache, &c.batch, prefix_table, prefix, (int32_t)max_q, max_length, (float)scale, c.dtype(), ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != WHT_OK) { Py_DECREF(out); Py_XDECREF(out_lse); return PyLong_FromLong(rc); }
    if (!lse) return out;
    PyObject* both = PyTuple_New(2);
    if (!both) { Py_DECREF(out); Py_DECREF(out_lse); return nullptr; }
    PyTuple_SET_ITEM(both, 0, out);
    PyTuple_SET_ITEM(both, 1, out_lse);
    return both;
    END_HANDLE_TH_ERRORS
}

// bind(addresses of wht_attention_append, wht_attention_workspace_bytes, wht_attention_paged, torch._C._cuda_getCurrentRawStream)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!expect(nargs, 4)) return nullptr;
    void* p[3];
    for (int i = 0; i < 3; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    lib_append = reinterpret_cast<decltype(lib_append)>(p[0]);
    lib_workspace_bytes = reinterpret_cast<decltype(lib_workspace_bytes)>(p[1]);
    lib_paged = reinterpret_cast<decltype(lib_paged)>(p[2]);
    Py_INCREF(args[3]);
    Py_XSETREF(raw_stream_of, args[3]);
    Py_RETURN_NONE;
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f))
PyMethodDef methods[] = {{"bind", FAST(bind), METH_FASTCALL, nullptr},
                         {"append", FAST(append), METH_FASTCALL, nullptr},
                         {"paged", FAST(paged), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_attention_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// torch_version: the torch this was compiled for (named by build.py); attention.py uses the module with no other.
PyMODINIT_FUNC PyInit__attention_marshal(void) {
    PyObject* m = PyModule_Create(&module_def);
    if (m && PyModule_AddStringConstant(m, "torch_version", WHT_TORCH_VERSION) < 0) Py_CLEAR(m);
    return m;
}

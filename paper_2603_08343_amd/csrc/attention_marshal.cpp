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
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/forward_grad.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/variable.h>

#include <cmath>

#include "../../include/wht_attention4.h"

namespace {

decltype(&wht_attention_append) lib_append;
decltype(&wht_attention_workspace_bytes) lib_workspace_bytes;
decltype(&wht_attention_paged) lib_paged;
decltype(&wht_attention_append4) lib_append4;
decltype(&wht_attention4_workspace_bytes) lib_workspace_bytes4;
decltype(&wht_attention_paged4) lib_paged4;
decltype(&wht_rotary_rotate) lib_rotate;
PyObject* raw_stream_of;                // torch._C._cuda_getCurrentRawStream
PyObject* general_rotate;               // autograd.WhtRotaryFunction.apply

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
    static bool is_plain(const at::Tensor& t) {
        static const c10::DispatchKeySet ordinary({c10::DispatchKey::CUDA, c10::DispatchKey::ADInplaceOrView,
                                                   c10::DispatchKey::AutogradCUDA, c10::DispatchKey::AutocastCUDA});
        return t.defined() && (t.key_set() | ordinary) == ordinary && t.is_cuda();
    }
    const at::Tensor* plain(PyObject* obj) {
        if (!THPVariable_CheckExact(obj)) return refuse();
        const at::Tensor& t = THPVariable_Unpack(obj);
        if (!is_plain(t)) return refuse();
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
    // The cache in 4 bits: codes and scales, each side alike.  The rows' type is `like`'s.
    wht_attention_cache4_t cache4{};
    void take_cache4(PyObject* const* args, PyObject* like) {
        if (modes_active()) { ok = false; return; }
        const at::Tensor *k = plain(args[0]), *v = plain(args[1]), *ks = plain(args[2]), *vs = plain(args[3]), *rows_like = plain(like);
        if (!ok) return;
        auto alike = [](const at::Tensor* a, const at::Tensor* b) {
            return a->dim() == 4 && b->dim() == 4 && a->sizes() == b->sizes() && a->strides() == b->strides() && a->scalar_type() == at::kByte &&
                   b->scalar_type() == at::kByte && a->device() == b->device() && a->numel() > 0;
        };
        if (!alike(k, v) || !alike(ks, vs) || k->device() != ks->device() || k->stride(3) != 1 || (ks->size(3) > 1 && ks->stride(3) != 1) || k->size(3) % 16 != 0 ||
            ks->size(3) != k->size(3) / 16) { ok = false; return; }
        for (int i = 0; i < 3; ++i)
            if (k->size(i) != ks->size(i) || k->size(i) > INT32_MAX) { ok = false; return; }
        take_type(rows_like);
        pages = k->size(0); heads = k->size(1); page_size = k->size(2); head_dim = 2 * k->size(3);
        if (!ok || device != k->device() || head_dim > INT32_MAX) { ok = false; return; }
        cache4 = {k->data_ptr(), v->data_ptr(), static_cast<uint8_t*>(ks->data_ptr()), static_cast<uint8_t*>(vs->data_ptr()),
                  k->stride(0), k->stride(1), k->stride(2), ks->stride(0), ks->stride(1), ks->stride(2),
                  (int32_t)pages, (int32_t)heads, (int32_t)page_size, (int32_t)head_dim};
    }
    // What the rows of a call are, by one of them; on the current device.
    void take_type(const at::Tensor* t) {
        type = t->scalar_type();
        device = t->device();
        const c10::impl::VirtualGuardImpl guard(c10::DeviceType::CUDA);
        if ((type != at::kFloat && type != at::kBFloat16) || guard.getDevice() != device) ok = false;
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

// What turns a call's heads: the table, positions [T] or [T][axes], the axis of each pair as bytes.
struct Angles {
    const float* rope = nullptr;
    int64_t rope_rows = 0, rotary = 0;
    const int32_t* positions = nullptr;
    int32_t axes = 1;
    const uint8_t* pair_axes = nullptr;
};
// Each is false for a tensor, or axes, that the library would read past, or as what they are not.
bool take_rope(Angles& a, const at::Tensor& r, c10::Device device) {
    if (!Call::is_plain(r) || r.scalar_type() != at::kFloat || r.dim() != 3 || r.size(2) != 2 || !r.is_contiguous() || r.device() != device || r.numel() == 0 ||
        r.size(1) > INT32_MAX / 2) return false;
    a.rope = static_cast<const float*>(r.data_ptr());
    a.rope_rows = r.size(0);
    a.rotary = 2 * r.size(1);
    return true;
}
bool take_positions(Angles& a, const at::Tensor& p, c10::Device device, int64_t T) {
    if (!Call::is_plain(p) || p.scalar_type() != at::kInt || p.dim() < 1 || p.dim() > 2 || p.size(0) != T || !p.is_contiguous() || p.device() != device ||
        (p.dim() == 2 && (p.size(1) < 1 || p.size(1) > WHT_ROTARY_MAX_AXES))) return false;
    a.positions = static_cast<const int32_t*>(p.data_ptr());
    a.axes = p.dim() == 2 ? (int32_t)p.size(1) : 1;
    return true;
}
bool take_axes(Angles& a, const char* axes, int64_t n) {
    if (n != a.rotary / 2) return false;
    a.pair_axes = reinterpret_cast<const uint8_t*>(axes);
    for (int64_t i = 0; i < n; ++i)
        if (a.pair_axes[i] >= a.axes) return false;
    return true;
}
void take_angles(Call& c, Angles& a, PyObject* rope, PyObject* positions, PyObject* axes, int64_t T) {
    if (!c.ok) return;
    if (rope != Py_None) {
        const at::Tensor* r = c.plain(rope);
        if (!r || !take_rope(a, *r, c.device)) { c.ok = false; return; }
    }
    if (positions != Py_None) {
        const at::Tensor* p = c.plain(positions);
        if (!p || !take_positions(a, *p, c.device, T)) { c.ok = false; return; }
    }
    if (axes != Py_None && (!PyBytes_CheckExact(axes) || !take_axes(a, PyBytes_AS_STRING(axes), PyBytes_GET_SIZE(axes)))) c.ok = false;
}

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

// What both attentions take: q, then table, lengths, q_starts | None, prefix_table | None, prefix_length, max_q | None, max_length | None, scale | None
// (args), and out | None, lse | None, want_lse, workspace | None.  The cache is taken.
template <class Bytes, class F>
PyObject* attend(Call& c, PyObject* q_obj, PyObject* const* args, PyObject* out_obj, PyObject* lse_obj, PyObject* want_obj, PyObject* ws_obj, Bytes lib_bytes, F&& call) {
    wht_attention_rows_t q{}, o{};
    const at::Tensor* qt = c.rows(q_obj, q, -1, -1);
    if (!c.ok) return none();
    const int64_t T = qt->size(0), q_heads = qt->size(1);
    c.take_batch(args[0], args[1], args[2], T);
    const int want_lse = PyObject_IsTrue(want_obj);
    if (want_lse < 0) return nullptr;
    const int64_t prefix = whole(args[4], 0, (int64_t)1 << 30, c.ok);
    const int32_t* prefix_table = nullptr;
    if (c.ok && prefix > 0) {
        if (args[3] == Py_None) return none();
        prefix_table = c.ints(args[3], 1, -1);
        if (!c.ok || THPVariable_Unpack(args[3]).size(0) < (prefix + c.page_size - 1) / c.page_size) return none();
    }
    const int64_t max_q = args[5] != Py_None ? whole(args[5], 1, INT32_MAX, c.ok) : c.batch.q_starts ? T : 1;
    const int64_t max_length = args[6] != Py_None ? whole(args[6], 0, INT64_MAX, c.ok) : (int64_t)c.batch.width * c.page_size;
    double scale = 1.0 / std::sqrt((double)c.head_dim);
    if (args[7] != Py_None) {
        if (!PyFloat_CheckExact(args[7])) return none();
        scale = PyFloat_AS_DOUBLE(args[7]);
    }
    if (c.ok && out_obj != Py_None) c.rows(out_obj, o, T, q_heads);
    float* lse = nullptr;
    if (c.ok && lse_obj != Py_None) {
        const at::Tensor* t = c.plain(lse_obj);
        if (!t || t->scalar_type() != at::kFloat || t->dim() != 2 || t->size(0) != T || t->size(1) != q_heads || !t->is_contiguous() || t->device() != c.device)
            return none();
        lse = static_cast<float*>(t->data_ptr());
    }
    if (!c.ok) return none();
    const size_t need = lib_bytes(T, c.batch.B, (int32_t)q_heads, (int32_t)c.heads, (int32_t)c.head_dim, (int32_t)max_q, max_length, prefix, c.dtype());
    void* ws = nullptr;
    size_t ws_bytes = 0;
    at::Tensor made_ws;
    if (ws_obj != Py_None) {
        const at::Tensor* t = c.plain(ws_obj);
        if (!t || !t->is_contiguous() || t->device() != c.device) return none();
        ws = t->data_ptr();
        ws_bytes = t->nbytes();
    } else if (need > 0) {
        made_ws = c.empty({(int64_t)need}, at::kByte);
        ws = made_ws.data_ptr();
        ws_bytes = need;
    }
    at::Tensor made_out, made_lse;
    if (out_obj == Py_None) {
        made_out = c.empty(qt->sizes(), c.type);
        o = {made_out.data_ptr(), made_out.stride(0), made_out.stride(1)};
    }
    if (!lse && want_lse) {
        made_lse = c.empty({T, q_heads}, at::kFloat);
        lse = static_cast<float*>(made_lse.data_ptr());
    }
    PyObject* out = made_out.defined() ? THPVariable_Wrap(std::move(made_out)) : Py_NewRef(out_obj);       // owned, both
    PyObject* out_lse = !lse ? nullptr : made_lse.defined() ? THPVariable_Wrap(std::move(made_lse)) : Py_NewRef(lse_obj);
    void* stream = nullptr;
    if (!out || (lse && !out_lse) || !c.stream(&stream)) { Py_XDECREF(out); Py_XDECREF(out_lse); return nullptr; }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call(&q, &o, lse, T, (int32_t)q_heads, prefix_table, prefix, (int32_t)max_q, max_length, (float)scale, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != WHT_OK) { Py_DECREF(out); Py_XDECREF(out_lse); return PyLong_FromLong(rc); }
    if (!lse) return out;
    PyObject* both = PyTuple_New(2);
    if (!both) { Py_DECREF(out); Py_DECREF(out_lse); return nullptr; }
    PyTuple_SET_ITEM(both, 0, out);
    PyTuple_SET_ITEM(both, 1, out_lse);
    return both;
}

// paged(q, k_pages, v_pages, table, lengths, q_starts | None, prefix_table | None, prefix_length, max_q | None, max_length | None, scale | None,
//       out | None, lse | None, want_lse, workspace | None)
PyObject* paged(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!expect(nargs, 15)) return nullptr;
    Call c;
    c.take_cache(args[1], args[2]);
    if (!c.ok) return none();
    return attend(c, args[0], args + 3, args[11], args[12], args[13], args[14], lib_workspace_bytes,
                  [&](const wht_attention_rows_t* q, const wht_attention_rows_t* o, float* lse, int64_t T, int32_t q_heads, const int32_t* prefix_table, int64_t prefix, int32_t max_q,
                      int64_t max_length, float scale, void* ws, size_t ws_bytes, void* stream) {
                      return lib_paged(q, o, lse, T, q_heads, &c.cache, &c.batch, prefix_table, prefix, max_q, max_length, scale, c.dtype(), ws, ws_bytes, stream);
                  });
    END_HANDLE_TH_ERRORS
}

// append4(q | None, k, v, k_pages, v_pages, k_scales, v_scales, table, lengths, rope | None, q_starts | None, position, positions | None, axes | None,
//         interleaved, transform, q_out | None, k_out | None, v_out | None, want_values)
PyObject* append4(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!expect(nargs, 20)) return nullptr;
    Call c;
    c.take_cache4(args + 3, args[1]);
    if (!c.ok) return none();
    wht_attention_rows_t q{}, k{}, v{}, out{}, k_out{}, v_out{};
    const at::Tensor* kt = c.rows(args[1], k, -1, c.heads);
    if (!c.ok) return none();
    const int64_t T = kt->size(0);
    c.rows(args[2], v, T, c.heads);
    const at::Tensor* qt = args[0] == Py_None ? nullptr : c.rows(args[0], q, T, -1);
    c.take_batch(args[7], args[8], args[10], T);
    const int64_t position = whole(args[11], 0, INT64_MAX, c.ok);
    Angles a;
    take_angles(c, a, args[9], args[12], args[13], T);
    const int interleaved = PyObject_IsTrue(args[14]), transform = PyObject_IsTrue(args[15]), want = PyObject_IsTrue(args[19]);
    if (interleaved < 0 || transform < 0 || want < 0) return nullptr;
    if ((args[17] == Py_None) != (args[18] == Py_None)) return none();
    if (qt && args[16] != Py_None) c.rows(args[16], out, T, qt->size(1));
    if (args[17] != Py_None) {
        c.rows(args[17], k_out, T, c.heads);
        c.rows(args[18], v_out, T, c.heads);
    }
    if (!c.ok) return none();
    PyObject *result = nullptr, *k_result = nullptr, *v_result = nullptr;                                    // owned
    auto make = [&](c10::IntArrayRef sizes, wht_attention_rows_t& r) {
        at::Tensor t = c.empty(sizes, c.type);
        r = {t.data_ptr(), t.stride(0), t.stride(1)};
        return THPVariable_Wrap(std::move(t));
    };
    const bool values = want || args[17] != Py_None;
    result = !qt ? Py_NewRef(Py_None) : args[16] != Py_None ? Py_NewRef(args[16]) : make(qt->sizes(), out);
    if (values) {
        k_result = args[17] != Py_None ? Py_NewRef(args[17]) : make(kt->sizes(), k_out);
        v_result = args[18] != Py_None ? Py_NewRef(args[18]) : make(kt->sizes(), v_out);
    }
    void* stream = nullptr;
    auto drop = [&]() { Py_XDECREF(result); Py_XDECREF(k_result); Py_XDECREF(v_result); };
    if (!result || (values && (!k_result || !v_result)) || !c.stream(&stream)) { drop(); return nullptr; }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = lib_append4(&q, &k, &v, &out, &k_out, &v_out, T, qt ? (int32_t)qt->size(1) : 0, &c.cache4, &c.batch, a.rope, a.rope_rows, (int32_t)a.rotary, interleaved,
                     position, a.positions, a.axes, a.pair_axes, transform, c.dtype(), stream);
    Py_END_ALLOW_THREADS
    if (rc != WHT_OK) { drop(); return PyLong_FromLong(rc); }
    if (values) {
        PyObject* all = PyTuple_New(3);
        if (!all) { drop(); return nullptr; }
        PyTuple_SET_ITEM(all, 0, result);
        PyTuple_SET_ITEM(all, 1, k_result);
        PyTuple_SET_ITEM(all, 2, v_result);
        return all;
    }
    // None would say that the call was declined
    if (!qt) { Py_DECREF(result); return PyTuple_New(0); }
    return result;
    END_HANDLE_TH_ERRORS
}

// paged4(q, k_pages, v_pages, k_scales, v_scales, table, lengths, q_starts | None, prefix_table | None, prefix_length, max_q | None, max_length | None,
//        scale | None, transform, out | None, lse | None, want_lse, workspace | None)
PyObject* paged4(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!expect(nargs, 18)) return nullptr;
    Call c;
    c.take_cache4(args + 1, args[0]);
    if (!c.ok) return none();
    const int transform = PyObject_IsTrue(args[13]);
    if (transform < 0) return nullptr;
    return attend(c, args[0], args + 5, args[14], args[15], args[16], args[17], lib_workspace_bytes4,
                  [&](const wht_attention_rows_t* q, const wht_attention_rows_t* o, float* lse, int64_t T, int32_t q_heads, const int32_t* prefix_table, int64_t prefix, int32_t max_q,
                      int64_t max_length, float scale, void* ws, size_t ws_bytes, void* stream) {
                      return lib_paged4(q, o, lse, T, q_heads, &c.cache4, &c.batch, prefix_table, prefix, max_q, max_length, scale, transform, c.dtype(), ws, ws_bytes, stream);
                  });
    END_HANDLE_TH_ERRORS
}

// rotate(x, rope, positions | None, axes | None, interleaved, inverse, out | None)
PyObject* rotate(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!expect(nargs, 7)) return nullptr;
    Call c;
    if (modes_active()) return none();
    const at::Tensor* x = c.plain(args[0]);
    if (!c.ok || x->dim() != 3 || x->numel() == 0 || x->size(2) > INT32_MAX || args[1] == Py_None) return none();
    c.take_type(x);
    c.head_dim = x->size(2);
    const int64_t T = x->size(0);
    wht_attention_rows_t in{}, out{};
    c.rows(args[0], in, T, -1);
    Angles a;
    take_angles(c, a, args[1], args[2], args[3], T);
    const int interleaved = PyObject_IsTrue(args[4]), inverse = PyObject_IsTrue(args[5]);
    if (interleaved < 0 || inverse < 0) return nullptr;
    if (c.ok && args[6] != Py_None) c.rows(args[6], out, T, x->size(1));
    if (!c.ok) return none();
    PyObject* result = nullptr;                                     // owned
    if (args[6] != Py_None) result = Py_NewRef(args[6]);
    else {
        at::Tensor t = c.empty(x->sizes(), c.type);
        out = {t.data_ptr(), t.stride(0), t.stride(1)};
        result = THPVariable_Wrap(std::move(t));
    }
    void* stream = nullptr;
    if (!result || !c.stream(&stream)) { Py_XDECREF(result); return nullptr; }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = lib_rotate(&in, &out, T, (int32_t)x->size(1), (int32_t)c.head_dim, a.rope, a.rope_rows, (int32_t)a.rotary, interleaved, a.positions, a.axes, a.pair_axes,
                    inverse, c.dtype(), stream);
    Py_END_ALLOW_THREADS
    if (rc != WHT_OK) { Py_DECREF(result); return PyLong_FromLong(rc); }
    return result;
    END_HANDLE_TH_ERRORS
}

struct Declined {};                     // the library refused the call: rotary.py's code says why

// The rotation of x [..., heads, head_dim]; nothing where a plain call does not do it.  The table and the positions are looked over each time: of a backward pass
// they are what a graph's hooks for saved tensors made of them.
at::Tensor turned(const at::Tensor& x, const at::Tensor& rope, const at::Tensor& positions, const std::string& axes, bool interleaved, bool inverse) {
    const int64_t D = x.size(-1), heads = x.size(-2), T = x.numel() / (heads * D), step = 16 / (int64_t)x.element_size();
    Angles a;
    if (!take_rope(a, rope, x.device()) || (positions.defined() && !take_positions(a, positions, x.device(), T)) ||
        (!axes.empty() && !take_axes(a, axes.data(), (int64_t)axes.size()))) return {};
    at::Tensor rows = x.reshape({T, heads, D});
    if (rows.stride(2) != 1 || rows.stride(1) % step != 0 || rows.stride(0) % step != 0 || rows.stride(1) < D || ((uintptr_t)rows.data_ptr() & 15u) != 0)
        rows = rows.clone(at::MemoryFormat::Contiguous);            // strides that the library does not take
    const at::Tensor y = at::cuda::empty(x.sizes(), x.options());
    const wht_attention_rows_t in{rows.data_ptr(), rows.stride(0), rows.stride(1)}, out{y.data_ptr(), heads * D, D};
    Call c;
    c.device = x.device();
    void* stream = nullptr;
    {
        const PyGILState_STATE gil = PyGILState_Ensure();
        const bool found = c.stream(&stream);
        if (!found) PyErr_Clear();
        PyGILState_Release(gil);
        if (!found) return {};
    }
    const int rc = lib_rotate(&in, &out, T, (int32_t)heads, (int32_t)D, a.rope, a.rope_rows, (int32_t)a.rotary, interleaved, a.positions, a.axes, a.pair_axes, inverse,
                              x.scalar_type() == at::kFloat ? WHT_DTYPE_F32 : WHT_DTYPE_BF16, stream);
    return rc == WHT_OK ? y : at::Tensor();
}

}  // namespace

// autograd.wht_rotary as a node of torch's C++ autograd (autograd.WhtRotaryFunction says what it does).  Forward and gradient of a step by
// torch.autograd.grad, of the host's time: 38.6 us as a Python Function, 31.7 here, a product by a constant 24.0.
// (named: the graph's nodes and torch's error messages show the type)
struct WhtRotaryFunction : torch::autograd::Function<WhtRotaryFunction> {
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& rope, const std::optional<at::Tensor>& given, const std::string& axes,
                              bool interleaved, bool inverse) {
        const at::Tensor positions = given ? *given : at::Tensor();
        const at::Tensor y = turned(x, rope, positions, axes, interleaved, inverse);
        if (!y.defined()) throw Declined{};
        ctx->save_for_backward({rope, positions});                  // their versions are checked: angles that have changed since raise
        ctx->saved_data["axes"] = axes;
        ctx->saved_data["interleaved"] = interleaved;
        ctx->saved_data["inverse"] = inverse;
        return y;
    }
    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, const torch::autograd::variable_list& grads) {
        const auto saved = ctx->get_saved_variables();
        const at::Tensor& dy = grads[0];
        const std::string& axes = ctx->saved_data["axes"].toStringRef();
        const bool interleaved = ctx->saved_data["interleaved"].toBool(), inverse = !ctx->saved_data["inverse"].toBool();
        torch::autograd::variable_list out(6);
        const c10::impl::VirtualGuardImpl guard(c10::DeviceType::CUDA);
        const bool ordinary = !modes_active() && Call::is_plain(dy) && (dy.scalar_type() == at::kFloat || dy.scalar_type() == at::kBFloat16) && guard.getDevice() == dy.device();
        if (ordinary && at::GradMode::is_enabled()) {               // a gradient of the gradient is asked for
            try {
                out[0] = apply(dy, saved[0], saved[1].defined() ? std::optional<at::Tensor>(saved[1]) : std::nullopt, axes, interleaved, inverse);
                return out;
            } catch (const Declined&) {
            }
        } else if (ordinary) out[0] = turned(dy, saved[0], saved[1], axes, interleaved, inverse);
        if (!out[0].defined()) out[0] = general(dy, saved[0], saved[1], axes, interleaved, inverse);
        return out;
    }
    // general_rotate(dy, rope, positions, axes, interleaved, inverse): autograd.WhtRotaryFunction.apply
    static at::Tensor general(const at::Tensor& dy, const at::Tensor& rope, const at::Tensor& positions, const std::string& axes, bool interleaved, bool inverse) {
        const PyGILState_STATE gil = PyGILState_Ensure();
        PyObject* args[6] = {THPVariable_Wrap(dy), THPVariable_Wrap(rope), positions.defined() ? THPVariable_Wrap(positions) : Py_NewRef(Py_None),
                             axes.empty() ? Py_NewRef(Py_None) : PyBytes_FromStringAndSize(axes.data(), (Py_ssize_t)axes.size()), PyBool_FromLong(interleaved), PyBool_FromLong(inverse)};
        PyObject* result = nullptr;
        if (args[0] && args[1] && args[2] && args[3]) result = PyObject_Vectorcall(general_rotate, args, 6, nullptr);
        for (PyObject* a : args) Py_XDECREF(a);
        at::Tensor dx;
        if (result && THPVariable_Check(result)) dx = THPVariable_Unpack(result);
        else if (result) PyErr_SetString(PyExc_TypeError, "wht_rotary_rotate returns a tensor");
        Py_XDECREF(result);
        python_error error;
        if (!dx.defined()) error.persist();
        PyGILState_Release(gil);
        if (!dx.defined()) throw error;
        return dx;
    }
};

namespace {

// rotary(x, rope, positions | None, axes | None, interleaved)
PyObject* rotary(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!expect(nargs, 5)) return nullptr;
    // transforms, traces and modes are keys that the thread includes beyond the ordinary ones
    if (modes_active() || c10::impl::tls_local_dispatch_key_set().included_ != c10::default_included_set ||
        torch::autograd::ForwardADLevel::try_get_by_idx(0)) return none();
    Call c;
    const at::Tensor* x = c.plain(args[0]);
    if (!c.ok || x->dim() < 3 || x->numel() == 0 || x->size(-1) > INT32_MAX || x->size(-2) > INT32_MAX || args[1] == Py_None) return none();
    c.take_type(x);
    const int64_t T = x->numel() / (x->size(-1) * x->size(-2));
    Angles a;
    take_angles(c, a, args[1], args[2], args[3], T);
    const int interleaved = PyObject_IsTrue(args[4]);
    if (interleaved < 0) return nullptr;
    if (!c.ok) return none();
    const std::string axes = a.pair_axes ? std::string(reinterpret_cast<const char*>(a.pair_axes), a.rotary / 2) : std::string();
    const std::optional<at::Tensor> positions = a.positions ? std::optional<at::Tensor>(THPVariable_Unpack(args[2])) : std::nullopt;
    try {
        return THPVariable_Wrap(WhtRotaryFunction::apply(*x, THPVariable_Unpack(args[1]), positions, axes, interleaved != 0, false));
    } catch (const Declined&) {
        return none();
    }
    END_HANDLE_TH_ERRORS
}

// leaf_elsewhere(x): whether a call would record a gradient for x that a living graph gathers on another stream than the current one.
PyObject* leaf_elsewhere(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (!expect(nargs, 1)) return nullptr;
    if (!THPVariable_Check(args[0]) || !at::GradMode::is_enabled()) Py_RETURN_FALSE;
    const at::Tensor& x = THPVariable_Unpack(args[0]);
    if (!x.is_cuda() || !x.requires_grad() || !x.is_leaf()) Py_RETURN_FALSE;
    const auto node = torch::autograd::impl::try_get_grad_accumulator(x);
    if (!node) Py_RETURN_FALSE;
    const auto stream = node->stream();
    const c10::impl::VirtualGuardImpl guard(c10::DeviceType::CUDA);
    return PyBool_FromLong(!stream || *stream != guard.getStream(x.device()));
    END_HANDLE_TH_ERRORS
}

// bind4(addresses of wht_attention_append4, wht_attention4_workspace_bytes, wht_attention_paged4, wht_rotary_rotate; autograd.WhtRotaryFunction.apply)
PyObject* bind4(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (!expect(nargs, 5)) return nullptr;
    void* p[4];
    for (int i = 0; i < 4; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    lib_append4 = reinterpret_cast<decltype(lib_append4)>(p[0]);
    lib_workspace_bytes4 = reinterpret_cast<decltype(lib_workspace_bytes4)>(p[1]);
    lib_paged4 = reinterpret_cast<decltype(lib_paged4)>(p[2]);
    lib_rotate = reinterpret_cast<decltype(lib_rotate)>(p[3]);
    Py_INCREF(args[4]);
    Py_XSETREF(general_rotate, args[4]);
    Py_RETURN_NONE;
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
                         {"bind4", FAST(bind4), METH_FASTCALL, nullptr},
                         {"append4", FAST(append4), METH_FASTCALL, nullptr},
                         {"paged4", FAST(paged4), METH_FASTCALL, nullptr},
                         {"rotate", FAST(rotate), METH_FASTCALL, nullptr},
                         {"rotary", FAST(rotary), METH_FASTCALL, nullptr},
                         {"leaf_elsewhere", FAST(leaf_elsewhere), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_attention_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// torch_version: the torch this was compiled for (named by build.py); attention.py uses the module with no other.
PyMODINIT_FUNC PyInit__attention_marshal(void) {
    PyObject* m = PyModule_Create(&module_def);
    if (m && PyModule_AddStringConstant(m, "torch_version", WHT_TORCH_VERSION) < 0) Py_CLEAR(m);
    return m;
}

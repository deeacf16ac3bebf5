// Argument marshalling of the per-token and per-prompt entry points for Python, as a CPython extension (module _native).
// A decode step of a few rows takes the GPU about as long as filling a ctypes structure takes the interpreter: reading
// data pointers, shapes and the current stream through the C++ side of torch costs well under a microsecond per call
// (a decode step of one row, back to back: 10.7 us through ctypes).
// Nothing is computed here; every function fills the argument structure of include/dsla.h, calls the C
// entry point of the same name and returns its status.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <initializer_list>

#include "dsla.h"

namespace {

// The tensor behind a Python argument: nullptr for None (and with an exception set for anything else).
struct Arg {
    const at::Tensor* t = nullptr;
    void* ptr = nullptr;
};
bool read_tensor(PyObject* o, Arg* out) {
    if (o == Py_None) return true;
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a torch tensor or None, got %s", Py_TYPE(o)->tp_name);
        return false;
    }
    out->t = &THPVariable_Unpack(o);
    out->ptr = out->t->data_ptr();
    return true;
}
bool read_tensors(PyObject* const* args, int n, Arg* out) {
    for (int i = 0; i < n; ++i)
        if (!read_tensor(args[i], &out[i])) return false;
    return true;
}
bool has_dims(const Arg& a, int dims, const char* name) {
    if (a.t && a.t->dim() == dims) return true;
    PyErr_Format(PyExc_ValueError, "%s must be a tensor of %d dimensions", name, dims);
    return false;
}
bool has_dims_from(const Arg& a, int dims, const char* name) {      // further dimensions are the caller's business: only size(dims - 1) is read
    if (a.t && a.t->dim() >= dims) return true;
    PyErr_Format(PyExc_ValueError, "%s must be a tensor of at least %d dimensions", name, dims);
    return false;
}
bool read_dtype(const at::Tensor& t, dsla_dtype* out) {
    if (t.scalar_type() == at::kBFloat16) { *out = DSLA_BF16; return true; }
    if (t.scalar_type() == at::kFloat) { *out = DSLA_F32; return true; }
    PyErr_SetString(PyExc_KeyError, "the element type must be torch.float32 or torch.bfloat16");
    return false;
}
dsla_gate_layout layout_of(const Arg& gates, int scalar_dims) {
    return gates.t && gates.t->dim() == scalar_dims + 1 ? DSLA_GATE_PER_KEY_CHANNEL : DSLA_GATE_SCALAR;
}
bool read_int(PyObject* o, int* out) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) return false;
    if (v != (int)v) { PyErr_SetString(PyExc_OverflowError, "value does not fit a C int"); return false; }
    *out = (int)v;
    return true;
}
bool read_float(PyObject* o, float* out) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) return false;
    *out = (float)v;
    return true;
}
bool read_handle(PyObject* o, dsla_state** out) {
    *out = o == Py_None ? nullptr : static_cast<dsla_state*>(PyLong_AsVoidPtr(o));
    return !PyErr_Occurred();
}
bool read_stream(PyObject* o, void** out) {
    if (o == Py_None) *out = c10::cuda::getCurrentCUDAStream().stream();
    else *out = PyLong_AsVoidPtr(o);
    return !PyErr_Occurred();
}
bool count_is(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return false;
}
size_t nbytes_of(const Arg& a) { return a.t ? (size_t)a.t->numel() * (size_t)a.t->element_size() : 0; }

// Runs a C entry point without the interpreter lock (a launch can wait for room in the stream's queue).
template <typename F> PyObject* status_of(F call) {
    dsla_status rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

#define GUARD_BEGIN try {
#define GUARD_END                                      \
    } catch (const std::exception& e) {                \
        PyErr_SetString(PyExc_RuntimeError, e.what()); \
        return nullptr;                                \
    }

// decode_step(q, k, v, o, g_hist, g_rec, gamma, slots, row_mask, handle, scale, stream) -> status
PyObject* py_decode_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[9];
    dsla_state* st;
    void* stream;
    dsla_decode_args a;
    std::memset(&a, 0, sizeof(a));
    if (!count_is(n, 12) || !read_tensors(args, 9, t) || !has_dims(t[0], 3, "q") || !has_dims_from(t[2], 3, "v") ||
        !read_dtype(*t[0].t, &a.dtype) || !read_handle(args[9], &st) || !read_float(args[10], &a.scale) || !read_stream(args[11], &stream))
        return nullptr;
    a.q = t[0].ptr; a.k = t[1].ptr; a.v = t[2].ptr; a.o = t[3].ptr;
    a.g_hist = static_cast<float*>(t[4].ptr); a.g_rec = static_cast<float*>(t[5].ptr); a.gamma = static_cast<float*>(t[6].ptr);
    a.slots = static_cast<int32_t*>(t[7].ptr); a.row_mask = static_cast<uint8_t*>(t[8].ptr);
    a.B = (int)t[0].t->size(0); a.H = (int)t[0].t->size(1); a.d_k = (int)t[0].t->size(2); a.d_v = (int)t[2].t->size(2);
    a.gate_layout = layout_of(t[4], 2);
    return status_of([&] { return dsla_decode_step(&a, st, stream); });
    GUARD_END
}

// nstate_decode_step(q, k, v, o, gates, weights, slots, row_mask, handle, scale, stream) -> status
PyObject* py_nstate_decode_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[8];
    dsla_state* st;
    void* stream;
    dsla_nstate_decode_args a;
    std::memset(&a, 0, sizeof(a));
    if (!count_is(n, 11) || !read_tensors(args, 8, t) || !has_dims(t[0], 3, "q") || !has_dims_from(t[2], 3, "v") || !read_dtype(*t[0].t, &a.dtype) ||
        !read_handle(args[8], &st) || !read_float(args[9], &a.scale) || !read_stream(args[10], &stream))
        return nullptr;
    if (!t[4].t || t[4].t->dim() < 1) { PyErr_SetString(PyExc_ValueError, "gates must be a tensor"); return nullptr; }
    a.q = t[0].ptr; a.k = t[1].ptr; a.v = t[2].ptr; a.o = t[3].ptr;
    a.gates = static_cast<float*>(t[4].ptr); a.weights = static_cast<float*>(t[5].ptr);
    a.slots = static_cast<int32_t*>(t[6].ptr); a.row_mask = static_cast<uint8_t*>(t[7].ptr);
    a.B = (int)t[0].t->size(0); a.H = (int)t[0].t->size(1); a.d_k = (int)t[0].t->size(2); a.d_v = (int)t[2].t->size(2);
    a.n_states = (int)t[4].t->size(0);
    a.gate_layout = layout_of(t[4], 3);
    return status_of([&] { return dsla_nstate_decode_step(&a, st, stream); });
    GUARD_END
}

// prefill(q, k, v, o, g_hist, g_rec, gamma, cu_seqlens, slots, workspace, handle, N, T, max_seqlen, chunk, scale,
//         use_initial_state, impl, stream) -> status
PyObject* py_prefill(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[10];
    dsla_state* st;
    void* stream;
    int impl;
    dsla_prefill_args a;
    std::memset(&a, 0, sizeof(a));
    if (!count_is(n, 19) || !read_tensors(args, 10, t) || !has_dims(t[0], 3, "q") || !has_dims_from(t[2], 3, "v") || !read_dtype(*t[0].t, &a.dtype) ||
        !read_handle(args[10], &st) || !read_int(args[11], &a.N) || !read_int(args[12], &a.T) || !read_int(args[13], &a.max_seqlen) ||
        !read_int(args[14], &a.chunk) || !read_float(args[15], &a.scale) || !read_int(args[16], &a.use_initial_state) ||
        !read_int(args[17], &impl) || !read_stream(args[18], &stream))
        return nullptr;
    a.q = t[0].ptr; a.k = t[1].ptr; a.v = t[2].ptr; a.o = t[3].ptr;
    a.g_hist = static_cast<float*>(t[4].ptr); a.g_rec = static_cast<float*>(t[5].ptr); a.gamma = static_cast<float*>(t[6].ptr);
    a.cu_seqlens = static_cast<int32_t*>(t[7].ptr); a.slots = static_cast<int32_t*>(t[8].ptr);
    a.workspace = t[9].ptr; a.workspace_bytes = nbytes_of(t[9]);
    a.T_total = (int)t[0].t->size(0); a.H = (int)t[0].t->size(1); a.d_k = (int)t[0].t->size(2); a.d_v = (int)t[2].t->size(2);
    a.impl = static_cast<dsla_impl>(impl);
    a.gate_layout = layout_of(t[4], 2);
    return status_of([&] { return dsla_prefill(&a, st, stream); });
    GUARD_END
}

// Sizes, types and layouts of a prefill call, which is all that its workspace depends on.
bool read_sizes(PyObject* const* args, const Arg& q, const Arg& v, const Arg& cu, dsla_prefill_args* a) {
    if (!has_dims(q, 3, "q") || !has_dims_from(v, 3, "v") || !read_dtype(*q.t, &a->dtype) || !read_int(args[0], &a->N) || !read_int(args[1], &a->T) ||
        !read_int(args[2], &a->max_seqlen))
        return false;
    a->cu_seqlens = static_cast<int32_t*>(cu.ptr);
    a->T_total = (int)q.t->size(0); a->H = (int)q.t->size(1); a->d_k = (int)q.t->size(2); a->d_v = (int)v.t->size(2);
    a->scale = 1.f;
    return true;
}

// prefill_workspace(q, v, g_hist, cu_seqlens, N, T, max_seqlen, chunk, impl) -> bytes
PyObject* py_prefill_workspace(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[4];
    int impl;
    dsla_prefill_args a;
    std::memset(&a, 0, sizeof(a));
    if (!count_is(n, 9) || !read_tensors(args, 4, t) || !read_sizes(args + 4, t[0], t[1], t[3], &a) || !read_int(args[7], &a.chunk) || !read_int(args[8], &impl))
        return nullptr;
    a.impl = static_cast<dsla_impl>(impl);
    a.gate_layout = layout_of(t[2], 2);
    return PyLong_FromSize_t(dsla_prefill_workspace_bytes(&a));
    GUARD_END
}

// nstate_prefill_workspace(q, v, gates, cu_seqlens, N, T, max_seqlen, impl) -> bytes
PyObject* py_nstate_prefill_workspace(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[4];
    int impl;
    dsla_prefill_args s;
    std::memset(&s, 0, sizeof(s));
    if (!count_is(n, 8) || !read_tensors(args, 4, t) || !read_sizes(args + 4, t[0], t[1], t[3], &s) || !read_int(args[7], &impl)) return nullptr;
    if (!t[2].t || t[2].t->dim() < 1) { PyErr_SetString(PyExc_ValueError, "gates must be a tensor"); return nullptr; }
    dsla_nstate_prefill_args a;
    std::memset(&a, 0, sizeof(a));
    a.cu_seqlens = s.cu_seqlens; a.N = s.N; a.T = s.T; a.T_total = s.T_total; a.max_seqlen = s.max_seqlen;
    a.H = s.H; a.d_k = s.d_k; a.d_v = s.d_v; a.dtype = s.dtype; a.scale = 1.f;
    a.n_states = (int)t[2].t->size(0);
    a.impl = static_cast<dsla_impl>(impl);
    a.gate_layout = layout_of(t[2], 3);
    return PyLong_FromSize_t(dsla_nstate_prefill_workspace_bytes(&a));
    GUARD_END
}

// nstate_prefill(q, k, v, o, gates, weights, cu_seqlens, slots, workspace, handle, N, T, max_seqlen, scale,
//                use_initial_state, impl, stream) -> status
PyObject* py_nstate_prefill(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[9];
    dsla_state* st;
    void* stream;
    int impl;
    dsla_nstate_prefill_args a;
    std::memset(&a, 0, sizeof(a));
    if (!count_is(n, 17) || !read_tensors(args, 9, t) || !has_dims(t[0], 3, "q") || !has_dims_from(t[2], 3, "v") || !read_dtype(*t[0].t, &a.dtype) ||
        !read_handle(args[9], &st) || !read_int(args[10], &a.N) || !read_int(args[11], &a.T) || !read_int(args[12], &a.max_seqlen) ||
        !read_float(args[13], &a.scale) || !read_int(args[14], &a.use_initial_state) || !read_int(args[15], &impl) ||
        !read_stream(args[16], &stream))
        return nullptr;
    if (!t[4].t || t[4].t->dim() < 1) { PyErr_SetString(PyExc_ValueError, "gates must be a tensor"); return nullptr; }
    a.q = t[0].ptr; a.k = t[1].ptr; a.v = t[2].ptr; a.o = t[3].ptr;
    a.gates = static_cast<float*>(t[4].ptr); a.weights = static_cast<float*>(t[5].ptr);
    a.cu_seqlens = static_cast<int32_t*>(t[6].ptr); a.slots = static_cast<int32_t*>(t[7].ptr);
    a.workspace = t[8].ptr; a.workspace_bytes = nbytes_of(t[8]);
    a.T_total = (int)t[0].t->size(0); a.H = (int)t[0].t->size(1); a.d_k = (int)t[0].t->size(2); a.d_v = (int)t[2].t->size(2);
    a.n_states = (int)t[4].t->size(0);
    a.impl = static_cast<dsla_impl>(impl);
    a.gate_layout = layout_of(t[4], 3);
    return status_of([&] { return dsla_nstate_prefill(&a, st, stream); });
    GUARD_END
}

// gate_project(x, w, bias, g_hist, g_rec, stream) -> status
PyObject* py_gate_project(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[5];
    void* stream;
    dsla_gate_project_args a;
    std::memset(&a, 0, sizeof(a));
    if (!count_is(n, 6) || !read_tensors(args, 5, t) || !has_dims(t[0], 2, "x") || !has_dims_from(t[1], 1, "w") || !read_stream(args[5], &stream)) return nullptr;
    a.x = t[0].ptr; a.w = t[1].ptr; a.bias = static_cast<float*>(t[2].ptr);
    a.g_hist = static_cast<float*>(t[3].ptr); a.g_rec = static_cast<float*>(t[4].ptr);
    a.T = (int)t[0].t->size(0); a.D_model = (int)t[0].t->size(1); a.H = (int)(t[1].t->size(0) / 2);
    return status_of([&] { return dsla_gate_project(&a, stream); });
    GUARD_END
}

// ---- entry points whose tensors are checked here: element type, sizes, contiguity, device ----
bool is_laid_out(const Arg& a, at::ScalarType type, std::initializer_list<int64_t> sizes, const at::Tensor& with, const char* name, bool optional = false) {
    if (!a.t) {
        if (optional) return true;
        PyErr_Format(PyExc_ValueError, "%s is missing", name);
        return false;
    }
    if (a.t->scalar_type() != type || a.t->sizes() != at::IntArrayRef(sizes) || !a.t->is_contiguous() || a.t->device() != with.device()) {
        PyErr_Format(PyExc_ValueError, "%s has another element type, shape or device than the call's other tensors ask for, or is not contiguous", name);
        return false;
    }
    return true;
}
// A launch goes to the current device: pointers of another one, or of the host, would fault there.
bool on_current_device(const at::Tensor& t, const char* name) {
    if (t.is_cuda() && t.device().index() == c10::cuda::current_device()) return true;
    PyErr_Format(PyExc_ValueError, "%s must be on the current CUDA device", name);
    return false;
}
bool fits_int(const at::Tensor& t) {
    for (const int64_t n : t.sizes())
        if (n > 0x7fffffff) { PyErr_SetString(PyExc_OverflowError, "a dimension does not fit a C int"); return false; }
    return true;
}

// q, k [rows, H_qk, d]; v, o [rows, H, d]; gate, beta [rows, H]
bool delta_tensors(const Arg* t, dsla_dtype* dtype) {
    if (!has_dims(t[0], 3, "q") || !has_dims(t[2], 3, "v") || !read_dtype(*t[0].t, dtype) || !fits_int(*t[0].t) || !fits_int(*t[2].t)) return false;
    const at::Tensor &q = *t[0].t, &v = *t[2].t;
    const int64_t rows = q.size(0), Hq = q.size(1), d = q.size(2), H = v.size(1), dv = v.size(2);
    const at::ScalarType type = q.scalar_type();
    return is_laid_out(t[0], type, {rows, Hq, d}, q, "q") && is_laid_out(t[1], type, {rows, Hq, d}, q, "k") && is_laid_out(t[2], type, {rows, H, dv}, q, "v") &&
           is_laid_out(t[3], type, {rows, H, dv}, q, "o") && is_laid_out(t[4], at::kFloat, {rows, H}, q, "gate") && is_laid_out(t[5], at::kFloat, {rows, H}, q, "beta") &&
           on_current_device(q, "q");
}

// delta_decode_step(q, k, v, o, gate, beta, slots, row_mask, handle, scale, stream) -> status
PyObject* py_delta_decode_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[8];
    dsla_state* st;
    void* stream;
    dsla_delta_decode_args a;
    std::memset(&a, 0, sizeof(a));
    if (!count_is(n, 11) || !read_tensors(args, 8, t) || !delta_tensors(t, &a.dtype) || !read_handle(args[8], &st) || !read_float(args[9], &a.scale) ||
        !read_stream(args[10], &stream))
        return nullptr;
    const at::Tensor &q = *t[0].t, &v = *t[2].t;
    if (!is_laid_out(t[6], at::kInt, {q.size(0)}, q, "slots", true) || !is_laid_out(t[7], at::kByte, {q.size(0)}, q, "row_mask", true)) return nullptr;
    a.q = t[0].ptr; a.k = t[1].ptr; a.v = t[2].ptr; a.o = t[3].ptr;
    a.gate = static_cast<float*>(t[4].ptr); a.beta = static_cast<float*>(t[5].ptr);
    a.slots = static_cast<int32_t*>(t[6].ptr); a.row_mask = static_cast<uint8_t*>(t[7].ptr);
    a.B = (int)q.size(0); a.H_qk = (int)q.size(1); a.d_k = (int)q.size(2); a.H = (int)v.size(1); a.d_v = (int)v.size(2);
    return status_of([&] { return dsla_delta_decode_step(&a, st, stream); });
    GUARD_END
}

// delta_prefill(q, k, v, o, gate, beta, cu_seqlens, slots, workspace, handle, N, T, max_seqlen, scale, use_initial_state, impl, stream) -> status
PyObject* py_delta_prefill(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[9];
    dsla_state* st;
    void* stream;
    int impl;
    dsla_delta_prefill_args a;
    std::memset(&a, 0, sizeof(a));
    if (!count_is(n, 17) || !read_tensors(args, 9, t) || !delta_tensors(t, &a.dtype) || !read_handle(args[9], &st) || !read_int(args[10], &a.N) ||
        !read_int(args[11], &a.T) || !read_int(args[12], &a.max_seqlen) || !read_float(args[13], &a.scale) || !read_int(args[14], &a.use_initial_state) ||
        !read_int(args[15], &impl) || !read_stream(args[16], &stream))
        return nullptr;
    const at::Tensor &q = *t[0].t, &v = *t[2].t;
    if (!is_laid_out(t[6], at::kInt, {(int64_t)a.N + 1}, q, "cu_seqlens", true) || !is_laid_out(t[7], at::kInt, {a.N}, q, "slots", true)) return nullptr;
    if (t[8].t && (!t[8].t->is_contiguous() || t[8].t->device() != q.device())) {
        PyErr_SetString(PyExc_ValueError, "the workspace must be contiguous and on the device of the call's tensors");
        return nullptr;
    }
    a.q = t[0].ptr; a.k = t[1].ptr; a.v = t[2].ptr; a.o = t[3].ptr;
    a.gate = static_cast<float*>(t[4].ptr); a.beta = static_cast<float*>(t[5].ptr);
    a.cu_seqlens = static_cast<int32_t*>(t[6].ptr); a.slots = static_cast<int32_t*>(t[7].ptr);
    a.workspace = t[8].ptr; a.workspace_bytes = nbytes_of(t[8]);
    a.T_total = (int)q.size(0); a.H_qk = (int)q.size(1); a.d_k = (int)q.size(2); a.H = (int)v.size(1); a.d_v = (int)v.size(2);
    a.impl = static_cast<dsla_impl>(impl);
    return status_of([&] { return dsla_delta_prefill(&a, st, stream); });
    GUARD_END
}

// Rows of [heads, d] with heads and channels contiguous; *stride: elements between rows.
bool read_rows(const Arg& a, int64_t rows, int64_t heads, int64_t d, const at::Tensor& with, const char* name, long long* stride) {
    if (!a.t || a.t->dim() != 3 || a.t->scalar_type() != with.scalar_type() || a.t->size(0) != rows || a.t->size(1) != heads || a.t->size(2) != d ||
        a.t->device() != with.device() || (d > 1 && a.t->stride(2) != 1) || (heads > 1 && a.t->stride(1) != d)) {
        PyErr_Format(PyExc_ValueError, "%s must be [T, heads, d] of the call's element type and device, with contiguous heads and channels", name);
        return false;
    }
    *stride = rows > 1 ? (long long)a.t->stride(0) : (long long)(heads * d);
    return true;
}

// qk_norm_rope(q, k, q_out, k_out, q_weight, k_weight, positions, inv_freq, eps, norm, interleaved, stream) -> status
PyObject* py_qk_norm_rope(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[8];
    void* stream;
    int norm;
    dsla_qk_norm_rope_args a;
    std::memset(&a, 0, sizeof(a));
    if (!count_is(n, 12) || !read_tensors(args, 8, t) || !has_dims(t[0], 3, "q") || !has_dims(t[1], 3, "k") || !read_dtype(*t[0].t, &a.dtype) ||
        !fits_int(*t[0].t) || !fits_int(*t[1].t) || !read_float(args[8], &a.eps) || !read_int(args[9], &norm) || !read_int(args[10], &a.interleaved) ||
        !read_stream(args[11], &stream))
        return nullptr;
    const at::Tensor &q = *t[0].t, &k = *t[1].t;
    const int64_t T = q.size(0), H = q.size(1), Hk = k.size(1), d = q.size(2), half = t[7].t ? t[7].t->numel() : 0;
    if (!read_rows(t[0], T, H, d, q, "q", &a.q_stride) || !read_rows(t[1], T, Hk, d, q, "k", &a.k_stride) ||
        !read_rows(t[2], T, H, d, q, "q_out", &a.q_out_stride) || !read_rows(t[3], T, Hk, d, q, "k_out", &a.k_out_stride) ||
        !is_laid_out(t[4], at::kFloat, {d}, q, "q_weight", true) || !is_laid_out(t[5], at::kFloat, {d}, q, "k_weight", true) ||
        !is_laid_out(t[6], at::kInt, {T}, q, "positions", half == 0) || !is_laid_out(t[7], at::kFloat, {half}, q, "inv_freq", true) || !on_current_device(q, "q"))
        return nullptr;
    if (half > 0x3fffffff) { PyErr_SetString(PyExc_OverflowError, "a dimension does not fit a C int"); return nullptr; }
    a.q = t[0].ptr; a.k = t[1].ptr; a.q_out = t[2].ptr; a.k_out = t[3].ptr;
    a.q_weight = static_cast<float*>(t[4].ptr); a.k_weight = static_cast<float*>(t[5].ptr);
    a.positions = static_cast<int32_t*>(t[6].ptr); a.inv_freq = static_cast<float*>(t[7].ptr);
    a.T = (int)T; a.H = (int)H; a.H_k = (int)Hk; a.d = (int)d; a.rot = 2 * (int)half;
    a.norm = static_cast<dsla_norm>(norm);
    return status_of([&] { return dsla_qk_norm_rope(&a, stream); });
    GUARD_END
}

// state_copy(src_slots, dst_slots, handle, stream) -> status
PyObject* py_state_copy(PyObject*, PyObject* const* args, Py_ssize_t n) {
    GUARD_BEGIN
    Arg t[2];
    dsla_state* st;
    void* stream;
    if (!count_is(n, 4) || !read_tensors(args, 2, t) || !has_dims(t[0], 1, "src_slots") || !read_handle(args[2], &st) || !read_stream(args[3], &stream)) return nullptr;
    const at::Tensor& src = *t[0].t;
    if (!fits_int(src) || !is_laid_out(t[0], at::kInt, {src.size(0)}, src, "src_slots") || !is_laid_out(t[1], at::kInt, {src.size(0)}, src, "dst_slots") ||
        !on_current_device(src, "src_slots"))
        return nullptr;
    return status_of([&] { return dsla_state_copy(st, static_cast<int32_t*>(t[0].ptr), static_cast<int32_t*>(t[1].ptr), (int)src.size(0), stream); });
    GUARD_END
}

#define FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f))
PyMethodDef kMethods[] = {{"decode_step", FAST(py_decode_step), METH_FASTCALL, nullptr},
                          {"nstate_decode_step", FAST(py_nstate_decode_step), METH_FASTCALL, nullptr},
                          {"prefill", FAST(py_prefill), METH_FASTCALL, nullptr},
                          {"prefill_workspace", FAST(py_prefill_workspace), METH_FASTCALL, nullptr},
                          {"nstate_prefill_workspace", FAST(py_nstate_prefill_workspace), METH_FASTCALL, nullptr},
                          {"nstate_prefill", FAST(py_nstate_prefill), METH_FASTCALL, nullptr},
                          {"gate_project", FAST(py_gate_project), METH_FASTCALL, nullptr},
                          {"delta_decode_step", FAST(py_delta_decode_step), METH_FASTCALL, nullptr},
                          {"delta_prefill", FAST(py_delta_prefill), METH_FASTCALL, nullptr},
                          {"qk_norm_rope", FAST(py_qk_norm_rope), METH_FASTCALL, nullptr},
                          {"state_copy", FAST(py_state_copy), METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_native", "Argument marshalling of libdsla for torch tensors.", -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&kModule); }

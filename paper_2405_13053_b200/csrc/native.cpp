// The per-call half of the Python binding in native code: argument checks, result allocation and the call into the C
// ABI of include/meteora.h.
//
// A decode call is 11 - 16 us on the GPU; marshalling it through ctypes (a dozen attribute reads and tensor checks in
// Python, six tensor ops for the two views of the routing) took 26 us on the host, so a caller that does not capture
// CUDA graphs waited for Python, not for the kernel.  The checks, messages and results are those of binding.py's
// documented functions; nothing of the layer is computed here and nothing is kept between calls.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstring>
#include <stdexcept>
#include <string>
#include <vector>

#include "meteora.h"

namespace {

PyObject* g_error = nullptr;   // binding.MeteoraError, set by init()

// A Python exception is already set.
struct PySet {};

[[noreturn]] void fail(PyObject* type, const std::string& text) {
    PyErr_SetString(type, text.c_str());
    throw PySet{};
}

void check(int status, const char* where) {
    if (status == METEORA_OK) return;
    PyObject* e = PyObject_CallFunction(g_error, "is", status, where);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw PySet{};
}

// A call into the library with the GIL released, as ctypes makes it: a launch can block on a full queue and a copy of
// pageable memory does, and other Python threads go on meanwhile.  Arguments are worked out before (under the GIL); the
// caller's references keep their tensors.
template <class Call>
int released(Call&& call) {
    struct Gil {
        PyThreadState* state = PyEval_SaveThread();
        ~Gil() { PyEval_RestoreThread(state); }
    } gil;
    return call();
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, std::string(name) + " must be a torch.Tensor");
    return THPVariable_Unpack(o);
}

int64_t integer(PyObject* o) {
    const int64_t direct = PyLong_Check(o) ? PyLong_AsLongLong(o) : -1;
    if (PyLong_Check(o)) {
        if (direct == -1 && PyErr_Occurred()) throw PySet{};
        return direct;
    }
    PyObject* n = PyNumber_Long(o);
    if (!n) throw PySet{};
    const int64_t v = PyLong_AsLongLong(n);
    Py_DECREF(n);
    if (v == -1 && PyErr_Occurred()) throw PySet{};
    return v;
}

double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PySet{};
    return v;
}

void dims(const at::Tensor& t, int64_t n, const char* name) {
    if (t.dim() != n) fail(PyExc_ValueError, std::string(name) + ": expected " + std::to_string(n) + " dimensions, got " + std::to_string(t.dim()));
}

meteora_dtype_t dtype_code(const at::Tensor& t) {
    const auto st = t.scalar_type();
    if (st == at::kFloat) return METEORA_F32;
    if (st == at::kBFloat16) return METEORA_BF16;
    fail(PyExc_TypeError, std::string("unsupported dtype torch.") + c10::toString(st) + "; the layer runs in float32 or bfloat16");
}

std::string size_text(at::IntArrayRef s) {
    std::string out = "(";
    for (size_t i = 0; i < s.size(); ++i) out += (i ? ", " : "") + std::to_string(s[i]);
    return out + (s.size() == 1 ? ",)" : ")");
}

// A contiguous CUDA tensor of this shape and type, or an exception.
void* dev(const at::Tensor& t, at::IntArrayRef shape, at::ScalarType dt, const char* name) {
    if (!t.is_cuda() || !t.is_contiguous()) fail(PyExc_ValueError, std::string(name) + " must be a contiguous CUDA tensor");
    if (t.sizes() != shape || t.scalar_type() != dt)
        fail(PyExc_ValueError, std::string(name) + ": expected " + size_text(shape) + " " + c10::toString(dt) + ", got " +
                                   size_text(t.sizes()) + " " + c10::toString(t.scalar_type()));
    return t.data_ptr();
}
void* dev(PyObject* o, at::IntArrayRef shape, at::ScalarType dt, const char* name) { return dev(tensor(o, name), shape, dt, name); }

void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

at::Tensor empty(at::IntArrayRef shape, at::ScalarType dt, const at::Tensor& like) {
    return at::empty(shape, at::TensorOptions().dtype(dt).device(like.device()));
}

meteora_shape_t make_shape(int64_t T, int64_t d_in, int64_t d_out, int64_t N, int64_t r, int64_t k, meteora_dtype_t dt, double temperature) {
    return meteora_shape_t{(int)T, (int)d_in, (int)d_out, (int)N, (int)r, (int)k, dt, (float)temperature};
}

at::Tensor zeroed(size_t bytes, const at::Tensor& like, const char* where) {
    // (the header alone needs zeros: clearing all of it took 2 to 30 us of a decode call made without a workspace)
    if (bytes == 0) check(METEORA_ERR_INVALID_ARG, where);
    at::Tensor ws = empty({(int64_t)bytes}, at::kByte, like);
    void* const st = stream();
    check(released([&] { return meteora_workspace_init(ws.data_ptr(), st); }), where);
    return ws;
}

// A [T, k] tensor over 4-byte values inside `workspace`: shares its storage and version counter, as a view does.
at::Tensor view_of(const at::Tensor& workspace, const void* ptr, at::ScalarType dt, int64_t T, int64_t k) {
    const int64_t off = (const char*)ptr - (const char*)workspace.storage().data();
    if (off % 4 != 0) fail(PyExc_RuntimeError, "the workspace does not start on a 4-byte boundary of its storage");
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(workspace.storage()), workspace.key_set(),
                                                     c10::scalarTypeToTypeMeta(dt));
    impl->set_storage_offset(off / 4);
    const int64_t sizes[2] = {T, k};
    impl->set_sizes_contiguous(at::IntArrayRef(sizes, 2));
    impl->set_version_counter(workspace.unsafeGetTensorImpl()->version_counter());
    return at::Tensor(std::move(impl));
}

PyObject* wrap(const at::Tensor& t) {
    PyObject* o = THPVariable_Wrap(t);
    if (!o) throw PySet{};
    return o;
}

PyObject* keep(PyObject* o) {
    Py_INCREF(o);
    return o;
}

template <class... P>
PyObject* tuple(P... parts) {
    PyObject* out = PyTuple_Pack(sizeof...(P), parts...);
    (Py_DECREF(parts), ...);
    if (!out) throw PySet{};
    return out;
}

typedef PyObject* (*Body)(PyObject* const* a);

template <Body body, int n_args>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != n_args) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", n_args, nargs);
        return nullptr;
    }
    try {
        return body(args);
    } catch (const PySet&) {
        return nullptr;
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// (x, Wg, k, temperature, want_logits) -> (idx, w, logits or None)
PyObject* gate_topk(PyObject* const* a) {
    const at::Tensor &x = tensor(a[0], "x"), &Wg = tensor(a[1], "Wg");
    dims(x, 2, "x");
    dims(Wg, 2, "Wg");
    const int64_t T = x.size(0), d_in = x.size(1), N = Wg.size(0), k = integer(a[2]);
    const meteora_shape_t s = make_shape(T, d_in, 1, N, 1, k, dtype_code(x), real(a[3]));
    const bool want = PyObject_IsTrue(a[4]) == 1;
    void *px = dev(x, {T, d_in}, x.scalar_type(), "x"), *pg = dev(Wg, {N, d_in}, x.scalar_type(), "Wg");
    at::Tensor idx = empty({T, k}, at::kInt, x), w = empty({T, k}, at::kFloat, x), logits;
    if (want) logits = empty({T, N}, at::kFloat, x);
    int32_t* const pi = (int32_t*)idx.data_ptr();
    float *const pw = (float*)w.data_ptr(), *const pl = want ? (float*)logits.data_ptr() : nullptr;
    void* const st = stream();
    check(released([&] { return meteora_gate_topk(px, pg, &s, pi, pw, pl, st); }), "meteora_gate_topk");
    return tuple(wrap(idx), wrap(w), want ? wrap(logits) : keep(Py_None));
}

// (topk_idx, N) -> (counts, offsets, perm)
PyObject* route(PyObject* const* a) {
    const at::Tensor& idx = tensor(a[0], "topk_idx");
    dims(idx, 2, "topk_idx");
    const int64_t T = idx.size(0), k = idx.size(1), N = integer(a[1]);
    void* p = dev(idx, {T, k}, at::kInt, "topk_idx");
    at::Tensor counts = empty({N}, at::kInt, idx), offsets = empty({N + 1}, at::kInt, idx), perm = empty({T * k}, at::kInt, idx);
    int32_t *const pc = (int32_t*)counts.data_ptr(), *const po = (int32_t*)offsets.data_ptr(), *const pp = (int32_t*)perm.data_ptr();
    void* const st = stream();
    check(released([&] { return meteora_route((const int32_t*)p, (int)T, (int)k, (int)N, pc, po, pp, st); }), "meteora_route");
    return tuple(wrap(counts), wrap(offsets), wrap(perm));
}

// (x, A, B, topk_idx, topk_w, offsets, perm, workspace or out, static) -> delta
PyObject* lora_delta(PyObject* const* a) {
    const at::Tensor &x = tensor(a[0], "x"), &A = tensor(a[1], "A"), &B = tensor(a[2], "B"), &idx = tensor(a[3], "topk_idx");
    dims(x, 2, "x");
    dims(A, 3, "A");
    dims(B, 3, "B");
    dims(idx, 2, "topk_idx");
    const int64_t T = x.size(0), d_in = x.size(1), N = A.size(0), r = A.size(1), d_out = B.size(1), k = idx.size(1);
    const bool is_static = a[8] == Py_True;
    const meteora_shape_t s = make_shape(T, d_in, d_out, N, r, k, dtype_code(x), 1.0);
    const auto dt = x.scalar_type();
    at::Tensor ws, delta;
    if (is_static && a[7] != Py_None) delta = tensor(a[7], "out");
    if (!is_static) ws = a[7] == Py_None ? zeroed(meteora_workspace_bytes(&s), x, "meteora_workspace_bytes") : tensor(a[7], "workspace");
    if (!delta.defined()) delta = empty({T, d_out}, at::kFloat, x);
    const void *px = dev(x, {T, d_in}, dt, "x"), *pA = dev(A, {N, r, d_in}, dt, "A"), *pB = dev(B, {N, d_out, r}, dt, "B");
    const int32_t* pi = (const int32_t*)dev(idx, {T, k}, at::kInt, "topk_idx");
    const float* pw = (const float*)dev(a[4], {T, k}, at::kFloat, "topk_w");
    const int32_t* po = (const int32_t*)dev(a[5], {N + 1}, at::kInt, "offsets");
    const int32_t* pp = (const int32_t*)dev(a[6], {T * k}, at::kInt, "perm");
    float* const out = (float*)dev(delta, {T, d_out}, at::kFloat, "delta");
    void *const pws = is_static ? nullptr : ws.data_ptr(), *const st = stream();
    const size_t ws_bytes = is_static ? 0 : (size_t)ws.numel();
    check(released([&] {
              return is_static ? meteora_lora_delta_static(px, pA, pB, pi, pw, po, pp, &s, out, st)
                               : meteora_lora_delta(px, pA, pB, pi, pw, po, pp, &s, out, pws, ws_bytes, st);
          }),
          is_static ? "meteora_lora_delta_static" : "meteora_lora_delta");
    return wrap(delta);
}

// (x, W0, A, B, Wg, k, temperature, workspace, out, return_routing) -> y or (y, idx, w)
PyObject* linear_forward(PyObject* const* a) {
    const at::Tensor &x = tensor(a[0], "x"), &W0 = tensor(a[1], "W0"), &A = tensor(a[2], "A");
    dims(x, 2, "x");
    dims(A, 3, "A");
    if (W0.dim() < 1) dims(W0, 2, "W0");
    const int64_t T = x.size(0), d_in = x.size(1), d_out = W0.size(0), N = A.size(0), r = A.size(1), k = integer(a[5]);
    const meteora_shape_t s = make_shape(T, d_in, d_out, N, r, k, dtype_code(x), real(a[6]));
    const auto dt = x.scalar_type();
    at::Tensor made_ws, made_y;
    if (a[7] == Py_None) made_ws = zeroed(meteora_workspace_bytes(&s), x, "meteora_workspace_bytes");
    if (a[8] == Py_None) made_y = empty({T, d_out}, dt, x);
    const at::Tensor &ws = made_ws.defined() ? made_ws : tensor(a[7], "workspace"), &y = made_y.defined() ? made_y : tensor(a[8], "out");
    const void *px = dev(x, {T, d_in}, dt, "x"), *pW = dev(W0, {d_out, d_in}, dt, "W0"), *pA = dev(A, {N, r, d_in}, dt, "A"),
               *pB = dev(a[3], {N, d_out, r}, dt, "B"), *pG = dev(a[4], {N, d_in}, dt, "Wg");
    void *const py = dev(y, {T, d_out}, dt, "y"), *const pws = ws.data_ptr(), *const st = stream();
    const size_t ws_bytes = (size_t)ws.numel();
    check(released([&] { return meteora_linear_forward(px, pW, pA, pB, pG, &s, py, pws, ws_bytes, st); }), "meteora_linear_forward");
    PyObject* y_obj = made_y.defined() ? wrap(y) : keep(a[8]);
    if (PyObject_IsTrue(a[9]) != 1) return y_obj;
    int32_t* p_idx = nullptr;
    float* p_w = nullptr;
    check(meteora_workspace_routing(&s, ws.data_ptr(), &p_idx, &p_w), "meteora_workspace_routing");
    return tuple(y_obj, wrap(view_of(ws, p_idx, at::kInt, T, k)), wrap(view_of(ws, p_w, at::kFloat, T, k)));
}

// (x_host, W0, A, B, Wg, k, y_host, workspace, temperature) -> y_host
PyObject* linear_forward_host(PyObject* const* a) {
    const at::Tensor &x = tensor(a[0], "x_host"), &W0 = tensor(a[1], "W0"), &A = tensor(a[2], "A"), &y = tensor(a[6], "y_host"),
                     &ws = tensor(a[7], "workspace");
    dims(x, 2, "x_host");
    dims(A, 3, "A");
    if (W0.dim() < 1) dims(W0, 2, "W0");
    const int64_t T = x.size(0), d_in = x.size(1), d_out = W0.size(0), N = A.size(0), r = A.size(1), k = integer(a[5]);
    const auto dt = W0.scalar_type();
    const meteora_shape_t s = make_shape(T, d_in, d_out, N, r, k, dt == at::kFloat ? METEORA_F32 : METEORA_BF16, real(a[8]));
    for (int i = 0; i < 2; ++i) {
        const at::Tensor& t = i ? y : x;
        if (t.is_cuda() || !t.is_contiguous() || t.scalar_type() != dt)
            fail(PyExc_ValueError, std::string(i ? "y_host" : "x_host") + " must be a contiguous host tensor of dtype " + c10::toString(dt));
    }
    if (y.dim() != 2 || y.size(0) != T || y.size(1) != d_out) fail(PyExc_ValueError, "y_host has the wrong shape");
    const void *px = x.data_ptr(), *pW = dev(W0, {d_out, d_in}, dt, "W0"), *pA = dev(A, {N, r, d_in}, dt, "A"),
               *pB = dev(a[3], {N, d_out, r}, dt, "B"), *pG = dev(a[4], {N, d_in}, dt, "Wg");
    void *const py = y.data_ptr(), *const pws = ws.data_ptr(), *const st = stream();
    const size_t ws_bytes = (size_t)ws.numel();
    check(released([&] { return meteora_linear_forward_host(px, pW, pA, pB, pG, &s, py, pws, ws_bytes, st); }), "meteora_linear_forward_host");
    return keep(a[6]);
}

// (x, A, B, dy, topk_idx, topk_w, temperature, Bt, workspace) -> (dWg, dlogit)
PyObject* gate_backward(PyObject* const* a) {
    const at::Tensor &x = tensor(a[0], "x"), &A = tensor(a[1], "A"), &idx = tensor(a[4], "topk_idx");
    const bool bt = a[7] != Py_None;
    const at::Tensor& B = tensor(bt ? a[7] : a[2], bt ? "Bt" : "B");
    dims(x, 2, "x");
    dims(A, 3, "A");
    dims(B, 3, bt ? "Bt" : "B");
    dims(idx, 2, "topk_idx");
    const int64_t T = x.size(0), d_in = x.size(1), N = A.size(0), r = A.size(1), d_out = B.size(bt ? 2 : 1), k = idx.size(1);
    const auto dt = x.scalar_type();
    const meteora_shape_t s = make_shape(T, d_in, d_out, N, r, k, dt == at::kFloat ? METEORA_F32 : METEORA_BF16, real(a[6]));
    const size_t need = meteora_gate_backward_workspace_bytes(&s);
    if (need == 0) check(METEORA_ERR_INVALID_ARG, "meteora_gate_backward_workspace_bytes");
    at::Tensor ws = a[8] == Py_None ? empty({(int64_t)need}, at::kByte, x) : tensor(a[8], "workspace");
    at::Tensor dWg = empty({N, d_in}, at::kFloat, x), dlogit = empty({T, k}, at::kFloat, x);
    const void* pB = bt ? dev(B, {N, r, d_out}, dt, "Bt") : dev(B, {N, d_out, r}, dt, "B");
    const auto fn = bt ? meteora_gate_backward_bt : meteora_gate_backward;
    const void *px = dev(x, {T, d_in}, dt, "x"), *pA = dev(A, {N, r, d_in}, dt, "A"), *pdy = dev(a[3], {T, d_out}, dt, "dy");
    const int32_t* pi = (const int32_t*)dev(idx, {T, k}, at::kInt, "topk_idx");
    const float* pw = (const float*)dev(a[5], {T, k}, at::kFloat, "topk_w");
    float *const pl = (float*)dlogit.data_ptr(), *const pd = (float*)dWg.data_ptr();
    void *const pws = ws.data_ptr(), *const st = stream();
    const size_t ws_bytes = (size_t)ws.numel();
    check(released([&] { return fn(px, pA, pB, pdy, pi, pw, &s, pl, pd, pws, ws_bytes, st); }), "meteora_gate_backward");
    return tuple(wrap(dWg), wrap(dlogit));
}

// (x, W0s, As, Bs, Wgs, k, temperature, workspace, return_routing) -> [y] or ([y], [(idx, w)])
PyObject* linear_forward_group(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    dims(x, 2, "x");
    const int64_t T = x.size(0), d_in = x.size(1), k = integer(a[5]);
    const double temperature = real(a[6]);
    const meteora_dtype_t code = dtype_code(x);
    const auto dt = x.scalar_type();
    struct Held {                        // the four sequences, as tuples or lists whose items can be read directly
        PyObject* o[4] = {};
        ~Held() {
            for (PyObject* p : o) Py_XDECREF(p);
        }
    } seq;
    const char* names[4] = {"W0", "A", "B", "Wg"};
    for (int i = 0; i < 4; ++i)
        if (!(seq.o[i] = PySequence_Fast(a[1 + i], "expected a sequence of tensors"))) throw PySet{};
    const Py_ssize_t G = PySequence_Fast_GET_SIZE(seq.o[0]);
    for (int i = 1; i < 4; ++i)
        if (PySequence_Fast_GET_SIZE(seq.o[i]) < G) fail(PyExc_IndexError, "a list of the group is shorter than W0s");
    if (G == 0) fail(PyExc_IndexError, "an empty group");
    auto item = [&](int i, Py_ssize_t m) -> const at::Tensor& { return tensor(PySequence_Fast_GET_ITEM(seq.o[i], m), names[i]); };
    dims(item(1, 0), 3, "A");
    const int64_t N = item(1, 0).size(0), r = item(1, 0).size(1);
    std::vector<int> d_out(G);
    for (Py_ssize_t m = 0; m < G; ++m) {
        if (item(0, m).dim() < 1) dims(item(0, m), 2, "W0");
        d_out[m] = (int)item(0, m).size(0);
    }
    const meteora_shape_t s = make_shape(T, d_in, d_out[0], N, r, k, code, temperature);
    at::Tensor ws = a[7] == Py_None ? zeroed(meteora_group_workspace_bytes(&s, d_out.data(), (int)G), x, "meteora_group_workspace_bytes")
                                    : tensor(a[7], "workspace");
    std::vector<at::Tensor> ys(G), held;                             // (held: another thread may change the lists meanwhile)
    held.reserve(4 * G);
    std::vector<const void*> ptr[4];
    for (auto& p : ptr) p.resize(G);
    std::vector<void*> py(G);
    for (Py_ssize_t m = 0; m < G; ++m) {
        ys[m] = empty({T, d_out[m]}, dt, x);
        py[m] = ys[m].data_ptr();
        ptr[0][m] = dev(item(0, m), {d_out[m], d_in}, dt, "W0");
        ptr[1][m] = dev(item(1, m), {N, r, d_in}, dt, "A");
        ptr[2][m] = dev(item(2, m), {N, d_out[m], r}, dt, "B");
        ptr[3][m] = dev(item(3, m), {N, d_in}, dt, "Wg");
        for (int i = 0; i < 4; ++i) held.push_back(item(i, m));
    }
    const void* px = dev(x, {T, d_in}, dt, "x");
    void *const pws = ws.data_ptr(), *const st = stream();
    const size_t ws_bytes = (size_t)ws.numel();
    check(released([&] {
              return meteora_linear_forward_group(px, ptr[0].data(), ptr[1].data(), ptr[2].data(), ptr[3].data(), d_out.data(), (int)G, &s,
                                                  py.data(), pws, ws_bytes, st);
          }),
          "meteora_linear_forward_group");
    PyObject* out = PyList_New(G);
    if (!out) throw PySet{};
    for (Py_ssize_t m = 0; m < G; ++m) PyList_SET_ITEM(out, m, wrap(ys[m]));
    if (PyObject_IsTrue(a[8]) != 1) return out;
    PyObject* routing = PyList_New(G);
    if (!routing) throw PySet{};
    for (Py_ssize_t m = 0; m < G; ++m) {
        int32_t* p_idx = nullptr;
        float* p_w = nullptr;
        check(meteora_group_workspace_routing(&s, d_out.data(), (int)G, (int)m, ws.data_ptr(), &p_idx, &p_w), "meteora_group_workspace_routing");
        PyList_SET_ITEM(routing, m, tuple(wrap(view_of(ws, p_idx, at::kInt, T, k)), wrap(view_of(ws, p_w, at::kFloat, T, k))));
    }
    return tuple(out, routing);
}

// ---- operators on heads -------------------------------------------------------------------------------------------
// Their calls run on the device of their first tensor, on that device's current stream, whichever device is current.

void* stream_of(const at::Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.get_device()).stream(); }

const at::Tensor& cuda_tensor(PyObject* o, const char* name) {
    const at::Tensor& t = tensor(o, name);
    if (!t.is_cuda()) fail(PyExc_ValueError, std::string(name) + " must be a CUDA tensor");
    return t;
}

void same_device(const at::Tensor& t, const at::Tensor& first, const char* name) {
    if (!t.is_cuda() || t.get_device() != first.get_device()) fail(PyExc_ValueError, std::string(name) + " must be on the device of the first tensor");
}

// x[T, heads, head_dim] with the entries of a head contiguous; any strides of tokens and heads.
meteora_heads_t heads(const at::Tensor& t, int64_t T, int64_t H, int64_t D, at::ScalarType dt, const at::Tensor& first, const char* name) {
    same_device(t, first, name);
    if (t.dim() != 3 || t.size(0) != T || t.size(1) != H || t.size(2) != D || t.scalar_type() != dt)
        fail(PyExc_ValueError, std::string(name) + ": expected " + size_text({T, H, D}) + " " + c10::toString(dt) + ", got " + size_text(t.sizes()) + " " +
                                   c10::toString(t.scalar_type()));
    if (D > 1 && t.stride(2) != 1) fail(PyExc_ValueError, std::string(name) + ": the entries of a head must be contiguous");
    return meteora_heads_t{t.data_ptr(), t.stride(0), t.stride(1), (int)H};
}

// Sizes that the library takes as int.
int small(int64_t v, const char* name) {
    if (v < 0 || v > INT32_MAX) fail(PyExc_ValueError, std::string(name) + " is out of range");
    return (int)v;
}

// The rotary embedding (binding.MeteoraRotary, a buffer of the struct's bytes), or nullptr for None.
struct Rotary {
    meteora_rotary_t value;
    const meteora_rotary_t* ptr = nullptr;
    explicit Rotary(PyObject* o) {
        if (o == Py_None) return;
        Py_buffer b;
        if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) throw PySet{};
        const bool fits = b.len == (Py_ssize_t)sizeof(value);
        if (fits) memcpy(&value, b.buf, sizeof(value));
        PyBuffer_Release(&b);
        if (!fits) fail(PyExc_TypeError, "rot must come from meteora_rotary_init");
        ptr = &value;
    }
};

struct Positions {
    const void* ptr = nullptr;
    int wide = 0;
    Positions(PyObject* o, int64_t T, const at::Tensor& first, bool needed) {
        if (o == Py_None && !needed) return;
        const at::Tensor& t = tensor(o, "positions");
        same_device(t, first, "positions");
        wide = t.scalar_type() == at::kLong;
        ptr = dev(t, {T}, wide ? at::kLong : at::kInt, "positions");
    }
};

// q (and k, unless None) with results of their shapes.
struct QkPair {
    const at::Tensor& q;
    int64_t T, D;
    at::ScalarType dt;
    meteora_dtype_t code;
    bool has_k;
    at::Tensor out[2];
    meteora_heads_t in[2], to[2];
    QkPair(PyObject* qo, PyObject* ko, PyObject* out_q, PyObject* out_k) : q(cuda_tensor(qo, "q")) {
        dims(q, 3, "q");
        T = q.size(0), D = q.size(2), dt = q.scalar_type(), code = dtype_code(q), has_k = ko != Py_None;
        small(T, "T");
        in[0] = heads(q, T, q.size(1), D, dt, q, "q");
        if (has_k) {
            const at::Tensor& k = tensor(ko, "k");
            dims(k, 3, "k");
            in[1] = heads(k, T, k.size(1), D, dt, q, "k");
        } else if (out_k != Py_None) {
            fail(PyExc_ValueError, "out_k without k");
        }
        PyObject* const given[2] = {out_q, out_k};
        for (int i = 0; i < (has_k ? 2 : 1); ++i) {
            out[i] = given[i] != Py_None ? tensor(given[i], i ? "out_k" : "out_q") : empty({T, in[i].heads, D}, dt, q);
            to[i] = heads(out[i], T, in[i].heads, D, dt, q, i ? "out_k" : "out_q");
        }
    }
    PyObject* result(int i) const { return i && !has_k ? keep(Py_None) : wrap(out[i]); }
};

const void* gain_of(PyObject* o, int64_t D, at::ScalarType dt, const at::Tensor& first, const char* name) {
    const at::Tensor& t = tensor(o, name);
    same_device(t, first, name);
    return dev(t, {D}, dt, name);
}

// (q, k or None, positions, rot, inverse, out_q or None, out_k or None) -> (q', k' or None)
PyObject* rotary(PyObject* const* a) {
    const at::Tensor& first = cuda_tensor(a[0], "q");
    const c10::cuda::CUDAGuard guard(first.device());
    QkPair p(a[0], a[1], a[5], a[6]);
    const Positions pos(a[2], p.T, first, true);
    const Rotary rot(a[3]);
    const int inverse = PyObject_IsTrue(a[4]) == 1;
    void* const st = stream_of(first);
    check(released([&] {
              return meteora_rotary(&p.in[0], p.has_k ? &p.in[1] : nullptr, &p.to[0], p.has_k ? &p.to[1] : nullptr, pos.ptr, pos.wide, (int)p.T,
                                    (int)p.D, p.code, rot.ptr, inverse, st);
          }),
          "meteora_rotary");
    return tuple(p.result(0), p.result(1));
}

// (q, k or None, q_gain, k_gain, positions, rot or None, eps, out_q, out_k) -> (q', k' or None)
PyObject* head_norm_rotary(PyObject* const* a) {
    const at::Tensor& first = cuda_tensor(a[0], "q");
    const c10::cuda::CUDAGuard guard(first.device());
    QkPair p(a[0], a[1], a[7], a[8]);
    const Rotary rot(a[5]);
    const Positions pos(a[4], p.T, first, rot.ptr != nullptr);
    const void* gq = gain_of(a[2], p.D, p.dt, first, "q_gain");
    const void* gk = p.has_k ? gain_of(a[3], p.D, p.dt, first, "k_gain") : nullptr;
    const float eps = (float)real(a[6]);
    void* const st = stream_of(first);
    check(released([&] {
              return meteora_head_norm_rotary(&p.in[0], p.has_k ? &p.in[1] : nullptr, gq, gk, &p.to[0], p.has_k ? &p.to[1] : nullptr, pos.ptr,
                                              pos.wide, (int)p.T, (int)p.D, p.code, rot.ptr, eps, st);
          }),
          "meteora_head_norm_rotary");
    return tuple(p.result(0), p.result(1));
}

// (dq', dk' or None, q, k or None, q_gain, k_gain, positions, rot or None, eps, workspace) -> (dq, dk, dq_gain, dk_gain)
PyObject* head_norm_rotary_backward(PyObject* const* a) {
    const at::Tensor& first = cuda_tensor(a[2], "q");
    const c10::cuda::CUDAGuard guard(first.device());
    QkPair p(a[2], a[3], Py_None, Py_None);
    meteora_heads_t dy[2];
    dy[0] = heads(tensor(a[0], "dq"), p.T, p.in[0].heads, p.D, p.dt, first, "dq");
    if (p.has_k) dy[1] = heads(tensor(a[1], "dk"), p.T, p.in[1].heads, p.D, p.dt, first, "dk");
    const Rotary rot(a[7]);
    const Positions pos(a[6], p.T, first, rot.ptr != nullptr);
    const void* gq = gain_of(a[4], p.D, p.dt, first, "q_gain");
    const void* gk = p.has_k ? gain_of(a[5], p.D, p.dt, first, "k_gain") : nullptr;
    const float eps = (float)real(a[8]);
    const size_t need = meteora_head_norm_rotary_backward_workspace_bytes((int)p.T, p.in[0].heads, p.has_k ? p.in[1].heads : 0, (int)p.D);
    if (need == 0) check(METEORA_ERR_UNSUPPORTED_SHAPE, "meteora_head_norm_rotary_backward");
    at::Tensor ws = a[9] == Py_None ? empty({(int64_t)need}, at::kByte, first) : tensor(a[9], "workspace");
    same_device(ws, first, "workspace");
    if (!ws.is_contiguous()) fail(PyExc_ValueError, "workspace must be contiguous");
    at::Tensor dgq = empty({p.D}, at::kFloat, first), dgk;
    if (p.has_k) dgk = empty({p.D}, at::kFloat, first);
    float *const pq = (float*)dgq.data_ptr(), *const pk = p.has_k ? (float*)dgk.data_ptr() : nullptr;
    void *const pws = ws.data_ptr(), *const st = stream_of(first);
    const size_t bytes = ws.nbytes();
    check(released([&] {
              return meteora_head_norm_rotary_backward(&dy[0], p.has_k ? &dy[1] : nullptr, &p.in[0], p.has_k ? &p.in[1] : nullptr, gq, gk, &p.to[0],
                                                       p.has_k ? &p.to[1] : nullptr, pq, pk, pos.ptr, pos.wide, (int)p.T, (int)p.D, p.code, rot.ptr,
                                                       eps, pws, bytes, st);
          }),
          "meteora_head_norm_rotary_backward");
    return tuple(p.result(0), p.result(1), wrap(dgq), p.has_k ? wrap(dgk) : keep(Py_None));
}

// k_cache, v_cache [pages, kv_heads, page_size, head_dim], page_table [B, width], lengths [B], cu_tokens [B + 1] or None
struct PagedBatch {
    meteora_cache_t cache;
    meteora_batch_t batch;
    at::ScalarType dt;
    int64_t D;
    PagedBatch(PyObject* kc, PyObject* vc, PyObject* table, PyObject* lengths, PyObject* cu, int64_t T, int64_t prefix_len, const at::Tensor& first) {
        const at::Tensor &k = tensor(kc, "k_cache"), &v = tensor(vc, "v_cache"), &pt = tensor(table, "page_table"), &len = tensor(lengths, "lengths");
        dims(k, 4, "k_cache");
        dims(pt, 2, "page_table");
        dt = k.scalar_type();
        D = k.size(3);
        const int64_t B = pt.size(0);
        same_device(k, first, "k_cache");
        same_device(v, first, "v_cache");
        same_device(pt, first, "page_table");
        same_device(len, first, "lengths");
        cache.k = dev(k, k.sizes(), dt, "k_cache");
        cache.v = dev(v, k.sizes(), dt, "v_cache");
        cache.n_pages = k.size(0);
        cache.kv_heads = small(k.size(1), "k_cache");
        cache.page_size = small(k.size(2), "k_cache");
        cache.head_dim = small(D, "k_cache");
        cache.dtype = dtype_code(k);
        batch.T = small(T, "T");
        batch.B = small(B, "page_table");
        batch.table_width = small(pt.size(1), "page_table");
        batch.page_table = (const int32_t*)dev(pt, {B, pt.size(1)}, at::kInt, "page_table");
        batch.lengths = (const int32_t*)dev(len, {B}, at::kInt, "lengths");
        batch.cu_tokens = nullptr;
        if (cu != Py_None) {
            same_device(tensor(cu, "cu_tokens"), first, "cu_tokens");
            batch.cu_tokens = (const int32_t*)dev(cu, {B + 1}, at::kInt, "cu_tokens");
        }
        batch.prefix_len = small(prefix_len, "prefix_len");
        batch.prefix_pages = nullptr;
    }
    void prefix(PyObject* pages, const at::Tensor& first) {
        const int64_t need = cache.page_size > 0 ? ((int64_t)batch.prefix_len + cache.page_size - 1) / cache.page_size : 0;
        if (pages == Py_None) {
            if (need > 0) fail(PyExc_ValueError, "prefix_len without prefix_pages");
            return;
        }
        const at::Tensor& t = tensor(pages, "prefix_pages");
        same_device(t, first, "prefix_pages");
        dims(t, 1, "prefix_pages");
        if (t.size(0) < need) fail(PyExc_ValueError, "prefix_pages holds fewer pages than prefix_len takes");
        batch.prefix_pages = (const int32_t*)dev(t, t.sizes(), at::kInt, "prefix_pages");
    }
};

// (k, v, k_cache, v_cache, page_table, lengths, rot or None, cu_tokens or None, prefix_len, q or None, q_gain, k_gain, eps, out_q) -> q' or None
PyObject* cache_append(PyObject* const* a) {
    const at::Tensor &k = cuda_tensor(a[0], "k"), &v = tensor(a[1], "v");
    const c10::cuda::CUDAGuard guard(k.device());
    dims(k, 3, "k");
    const int64_t T = k.size(0);
    PagedBatch p(a[2], a[3], a[4], a[5], a[7], T, integer(a[8]), k);
    const Rotary rot(a[6]);
    const meteora_heads_t hk = heads(k, T, p.cache.kv_heads, p.D, p.dt, k, "k"), hv = heads(v, T, p.cache.kv_heads, p.D, p.dt, k, "v");
    meteora_heads_t hq, ho;
    at::Tensor out;
    const bool has_q = a[9] != Py_None;
    if (has_q) {
        const at::Tensor& q = tensor(a[9], "q");
        dims(q, 3, "q");
        hq = heads(q, T, q.size(1), p.D, p.dt, k, "q");
        out = a[13] != Py_None ? tensor(a[13], "out_q") : empty({T, q.size(1), p.D}, p.dt, k);
        ho = heads(out, T, q.size(1), p.D, p.dt, k, "out_q");
    } else if (a[13] != Py_None || a[10] != Py_None) {
        fail(PyExc_ValueError, "out_q and q_gain need q");
    }
    const void* gq = a[10] != Py_None ? gain_of(a[10], p.D, p.dt, k, "q_gain") : nullptr;
    const void* gk = a[11] != Py_None ? gain_of(a[11], p.D, p.dt, k, "k_gain") : nullptr;
    const float eps = (float)real(a[12]);
    void* const st = stream_of(k);
    check(released([&] {
              return meteora_cache_append(&hk, &hv, has_q ? &hq : nullptr, has_q ? &ho : nullptr, gq, gk, eps, rot.ptr, &p.cache, &p.batch, st);
          }),
          "meteora_cache_append");
    return has_q ? wrap(out) : keep(Py_None);
}

at::Tensor attention_workspace(const PagedBatch& p, int q_heads, const at::Tensor& first) {
    const size_t need = meteora_prefix_attention_workspace_bytes(&p.cache, &p.batch, q_heads);
    if (need == 0) check(METEORA_ERR_INVALID_ARG, "meteora_prefix_attention_workspace_bytes");
    at::Tensor ws = empty({(int64_t)need}, at::kByte, first);
    void* const st = stream_of(first);
    check(released([&] { return meteora_workspace_init(ws.data_ptr(), st); }), "meteora_workspace_init");
    return ws;
}

// (q, k_cache, v_cache, page_table, lengths, prefix_pages or None, prefix_len, cu_tokens or None, scale or None, workspace, out, return_lse)
PyObject* prefix_attention(PyObject* const* a) {
    const at::Tensor& q = cuda_tensor(a[0], "q");
    const c10::cuda::CUDAGuard guard(q.device());
    dims(q, 3, "q");
    const int64_t T = q.size(0), H = q.size(1);
    PagedBatch p(a[1], a[2], a[3], a[4], a[7], T, integer(a[6]), q);
    p.prefix(a[5], q);
    const meteora_heads_t hq = heads(q, T, H, p.D, p.dt, q, "q");
    at::Tensor made_ws, out = a[10] != Py_None ? tensor(a[10], "out") : empty({T, H, p.D}, p.dt, q), lse;
    const meteora_heads_t ho = heads(out, T, H, p.D, p.dt, q, "out");
    if (a[9] == Py_None) made_ws = attention_workspace(p, small(H, "q"), q);
    const at::Tensor& ws = made_ws.defined() ? made_ws : tensor(a[9], "workspace");
    same_device(ws, q, "workspace");
    if (!ws.is_contiguous()) fail(PyExc_ValueError, "workspace must be contiguous");
    const bool want_lse = PyObject_IsTrue(a[11]) == 1;
    if (want_lse) lse = empty({T, H}, at::kFloat, q);
    float* const pl = want_lse ? (float*)lse.data_ptr() : nullptr;
    const float scale = a[8] == Py_None ? (float)(1.0 / std::sqrt((double)p.D)) : (float)real(a[8]);
    void *const pws = ws.data_ptr(), *const st = stream_of(q);
    const size_t bytes = ws.nbytes();
    check(released([&] { return meteora_prefix_attention(&hq, &p.cache, &p.batch, scale, &ho, pl, pws, bytes, st); }), "meteora_prefix_attention");
    PyObject* out_obj = a[10] != Py_None ? keep(a[10]) : wrap(out);
    return want_lse ? tuple(out_obj, wrap(lse)) : out_obj;
}

PyObject* init(PyObject* const* a) {
    Py_XDECREF(g_error);
    g_error = keep(a[0]);
    return keep(Py_None);
}

#define METEORA_METHOD(name, n) {#name, (PyCFunction)(void (*)(void))entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METEORA_METHOD(gate_topk, 5),           METEORA_METHOD(route, 2),
                         METEORA_METHOD(lora_delta, 9),          METEORA_METHOD(linear_forward, 10),
                         METEORA_METHOD(linear_forward_host, 9), METEORA_METHOD(gate_backward, 9),
                         METEORA_METHOD(linear_forward_group, 9), METEORA_METHOD(init, 1),
                         METEORA_METHOD(rotary, 7),               METEORA_METHOD(head_norm_rotary, 9),
                         METEORA_METHOD(head_norm_rotary_backward, 10), METEORA_METHOD(cache_append, 14),
                         METEORA_METHOD(prefix_attention, 12),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&module); }

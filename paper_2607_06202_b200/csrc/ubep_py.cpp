// CPython module for the calls a layer makes every step: tensors and the current stream to the C ABI of
// libubep.so without going through ctypes.
//
// Why it exists: on a B200 host a decode-sized layer takes the GPU 8 to 25 us, and through ctypes the two
// calls took the host 20.4 us -- 3.6 us per call to ask torch for the current stream object, 0.2 us per
// pointer, 0.6 us for ctypes itself, 2.5 us for torch.empty -- against 2.6 to 2.9 us per kernel launch,
// which is what is left.  Nothing here is cached between calls.
//
// The library's entry points are handed over by address (bind), so this module links neither libubep.so
// nor the CUDA runtime.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <exception>

#include "../../include/ubep.h"

namespace {

decltype(&ubep_dispatch) f_dispatch;
decltype(&ubep_combine) f_combine;
decltype(&ubep_get_dispatch_layout) f_layout;
decltype(&ubep_dispatch_sync) f_dispatch_sync;
decltype(&ubep_route) f_route;
decltype(&ubep_route_backward) f_route_backward;
decltype(&ubep_expert_gated) f_gated;
decltype(&ubep_expert_gated_backward) f_gated_backward;
decltype(&ubep_expert_linear) f_linear;
decltype(&ubep_expert_linear_backward) f_linear_backward;

// An argument that must be a contiguous tensor, or None where the C ABI takes a null pointer.
bool tensor_arg(PyObject* o, void** ptr, const at::Tensor** t = nullptr) {
    if (o == Py_None) {
        *ptr = nullptr;
        return true;
    }
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a tensor or None, got %s", Py_TYPE(o)->tp_name);
        return false;
    }
    const at::Tensor& v = THPVariable_Unpack(o);
    if (!v.is_contiguous()) {
        PyErr_SetString(PyExc_AssertionError, "tensor is not contiguous");
        return false;
    }
    *ptr = v.data_ptr();
    if (t) *t = &v;
    return true;
}

bool rows_of(PyObject* o, int32_t* rows) {   // first dimension of a tensor
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a tensor, got %s", Py_TYPE(o)->tp_name);
        return false;
    }
    const at::Tensor& v = THPVariable_Unpack(o);
    if (v.dim() < 1) {
        PyErr_SetString(PyExc_IndexError, "tensor has no dimension");
        return false;
    }
    const int64_t n = v.size(0);
    *rows = n > INT32_MAX ? INT32_MAX : (int32_t)n;
    return true;
}

bool int_arg(PyObject* o, long long* v) {
    *v = PyLong_AsLongLong(o);
    return !(*v == -1 && PyErr_Occurred());
}

bool count_arg(PyObject* o, int32_t* v) {   // an int32 of the C ABI (out of range: an argument error there)
    long long n;
    if (!int_arg(o, &n)) return false;
    *v = n < INT32_MIN || n > INT32_MAX ? -1 : (int32_t)n;
    return true;
}

// The library's buffer handle as an integer; None after the buffer was closed.
bool handle_arg(PyObject* o, ubep_buffer_t** buf) {
    *buf = o == Py_None ? nullptr : static_cast<ubep_buffer_t*>(PyLong_AsVoidPtr(o));
    return !PyErr_Occurred();
}

// None = torch's current stream; otherwise an object with a `cuda_stream` handle, or the handle as anything int() takes.
bool stream_arg(PyObject* o, void** st) {
    if (o == Py_None) {
        *st = c10::cuda::getCurrentCUDAStream().stream();
        return true;
    }
    PyObject* h = nullptr;
    if (PyLong_Check(o)) {
        h = Py_NewRef(o);
    } else if (PyObject_HasAttrString(o, "cuda_stream")) {
        h = PyObject_GetAttrString(o, "cuda_stream");
    } else {
        h = PyNumber_Long(o);
    }
    if (!h) return false;
    *st = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    return !PyErr_Occurred();
}

// Memory for work on stream `st`, `current` being torch's.  It comes from the pool of `st` itself: the allocator hands a block out again
// as soon as it is given back, and only the stream it was given back on is sure to be done with it by then -- from the current
// stream's pool a kernel on another one would write what the current stream may still work on.  `kept`: the caller gets it, who
// may use it on the current stream as well, so what that has under way is waited for before the block goes to anybody else.
at::Tensor memory_on(void* st, const c10::cuda::CUDAStream& current, c10::IntArrayRef shape, at::ScalarType type, bool kept) {
    const c10::Device dev = current.device();
    if (st == static_cast<void*>(current.stream())) return at::detail::empty_cuda(shape, type, dev, c10::nullopt);
    if (st == reinterpret_cast<void*>(1)) st = nullptr;   // cudaStreamLegacy: the default stream by its other name
    const c10::cuda::CUDAStreamGuard on(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(st), dev.index()));
    at::Tensor t = at::detail::empty_cuda(shape, type, dev, c10::nullopt);
    if (kept) t.record_stream(current.unwrap());
    return t;
}

bool want_args(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return false;
}

PyObject* translate_exception() {
    try {
        throw;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// The GIL is released around a library call, as ctypes does: a launch may wait for room in the stream's queue.
template <typename F>
int without_gil(F call) {
    PyThreadState* state = PyEval_SaveThread();
    const int rc = call();
    PyEval_RestoreThread(state);
    return rc;
}

// Every call below returns an int (the C ABI's code) or, where it makes its outputs, those.

// dispatch(handle, x, topk_idx, topk_w, T or None, stream): T defaults to x's rows
PyObject* py_dispatch(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 6)) return nullptr;
        ubep_buffer_t* buf;
        void *x, *idx, *w, *st;
        int32_t T = 0;
        if (!handle_arg(a[0], &buf) || !tensor_arg(a[1], &x) || !tensor_arg(a[2], &idx) || !tensor_arg(a[3], &w) ||
            !(a[4] == Py_None ? rows_of(a[1], &T) : count_arg(a[4], &T)) || !stream_arg(a[5], &st))
            return nullptr;
        return PyLong_FromLong(without_gil([&] {
            return f_dispatch(buf, x, static_cast<const int32_t*>(idx), static_cast<const float*>(w), T, st);
        }));
    } catch (...) {
        return translate_exception();
    }
}

// dispatch_sync(handle, protocol, x, topk_idx, topk_w, T or None, stream)
PyObject* py_dispatch_sync(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 7)) return nullptr;
        ubep_buffer_t* buf;
        void *x, *idx, *w, *st;
        int32_t T = 0, proto;
        if (!handle_arg(a[0], &buf) || !count_arg(a[1], &proto) || !tensor_arg(a[2], &x) || !tensor_arg(a[3], &idx) ||
            !tensor_arg(a[4], &w) || !(a[5] == Py_None ? rows_of(a[2], &T) : count_arg(a[5], &T)) ||
            !stream_arg(a[6], &st))
            return nullptr;
        return PyLong_FromLong(without_gil([&] {
            return f_dispatch_sync(buf, proto, x, static_cast<const int32_t*>(idx), static_cast<const float*>(w), T, st);
        }));
    } catch (...) {
        return translate_exception();
    }
}

// combine(handle, y, topk_w, T or None, out, stream): T defaults to topk_w's rows; the code
PyObject* py_combine(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 6)) return nullptr;
        ubep_buffer_t* buf;
        void *y, *w, *out, *st;
        int32_t T = 0;
        if (!handle_arg(a[0], &buf) || !tensor_arg(a[1], &y) || !tensor_arg(a[2], &w) ||
            !(a[3] == Py_None ? rows_of(a[2], &T) : count_arg(a[3], &T)) || !tensor_arg(a[4], &out) ||
            !stream_arg(a[5], &st))
            return nullptr;
        return PyLong_FromLong(without_gil([&] {
            return f_combine(buf, y, static_cast<const float*>(w), T, out, st);
        }));
    } catch (...) {
        return translate_exception();
    }
}

// combine_new(handle, y, topk_w, hidden, device, stream): the bf16 output [rows of topk_w, hidden], or the code
PyObject* py_combine_new(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 6)) return nullptr;
        ubep_buffer_t* buf;
        void *y, *w, *st;
        int32_t T;
        long long hidden, device;
        if (!handle_arg(a[0], &buf) || !tensor_arg(a[1], &y) || !tensor_arg(a[2], &w) || !rows_of(a[2], &T) ||
            !int_arg(a[3], &hidden) || !int_arg(a[4], &device) || !stream_arg(a[5], &st))
            return nullptr;
        const auto current = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device);
        at::Tensor out = memory_on(st, current, {(int64_t)T, (int64_t)hidden}, at::kBFloat16, true);
        void* po = out.data_ptr();
        const int rc = without_gil([&] { return f_combine(buf, y, static_cast<const float*>(w), T, po, st); });
        if (rc != UBEP_OK) return PyLong_FromLong(rc);
        return THPVariable_Wrap(std::move(out));
    } catch (...) {
        return translate_exception();
    }
}

// layout(handle, topk_idx, T, tokens_per_rank, tokens_per_expert, is_token_in_rank, stream): the code
PyObject* py_layout(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 7)) return nullptr;
        ubep_buffer_t* buf;
        void *idx, *npr, *npe, *itr, *st;
        int32_t T;
        if (!handle_arg(a[0], &buf) || !tensor_arg(a[1], &idx) || !count_arg(a[2], &T) || !tensor_arg(a[3], &npr) ||
            !tensor_arg(a[4], &npe) || !tensor_arg(a[5], &itr) || !stream_arg(a[6], &st))
            return nullptr;
        return PyLong_FromLong(without_gil([&] {
            return f_layout(buf, static_cast<const int32_t*>(idx), T, static_cast<int32_t*>(npr),
                            static_cast<int32_t*>(npe), static_cast<uint8_t*>(itr), st);
        }));
    } catch (...) {
        return translate_exception();
    }
}

// layout_new(handle, topk_idx, num_ranks, num_experts, device, stream): the tuple (tokens_per_rank [R] int32,
// tokens_per_expert [E] int32, is_token_in_rank [T, R] uint8), or the code.  Three allocations: each result is a tensor of
// its own, which a caller may keep, save or resize without the others.
PyObject* py_layout_new(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 6)) return nullptr;
        ubep_buffer_t* buf;
        void *idx, *st;
        int32_t T;
        long long R, E, device;
        if (!handle_arg(a[0], &buf) || !tensor_arg(a[1], &idx) || !rows_of(a[1], &T) || !int_arg(a[2], &R) ||
            !int_arg(a[3], &E) || !int_arg(a[4], &device) || !stream_arg(a[5], &st))
            return nullptr;
        const auto current = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device);
        at::Tensor parts[3] = {memory_on(st, current, {(int64_t)R}, at::kInt, true), memory_on(st, current, {(int64_t)E}, at::kInt, true),
                               memory_on(st, current, {(int64_t)T, (int64_t)R}, at::kByte, true)};
        void* po[3] = {parts[0].data_ptr(), parts[1].data_ptr(), parts[2].data_ptr()};
        const int rc = without_gil([&] {
            return f_layout(buf, static_cast<const int32_t*>(idx), T, static_cast<int32_t*>(po[0]),
                            static_cast<int32_t*>(po[1]), static_cast<uint8_t*>(po[2]), st);
        });
        if (rc != UBEP_OK) return PyLong_FromLong(rc);
        PyObject* out = PyTuple_New(3);
        if (!out) return nullptr;
        for (int i = 0; i < 3; ++i) {
            PyObject* o = THPVariable_Wrap(std::move(parts[i]));
            if (!o) {
                Py_DECREF(out);
                return nullptr;
            }
            PyTuple_SET_ITEM(out, i, o);
        }
        return out;
    } catch (...) {
        return translate_exception();
    }
}

// ------------------------------------------------------------------ router and experts
//
// These calls take their sizes from the tensors, so they hold every tensor against them: a wrong type or shape raises a
// ValueError that names the argument, and nothing is launched.

struct Refused : std::exception {
    char text[160];
    Refused(const char* name, const char* what) { std::snprintf(text, sizeof text, "%s: %s", name, what); }
    const char* what() const noexcept override { return text; }
};
struct Raised : std::exception {};   // the Python error is set

PyObject* refused_or_raised() {
    try {
        throw;
    } catch (const Raised&) {
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// Where the tensors of a call live and which stream it runs on.
struct Place {
    c10::Device dev;
    c10::cuda::CUDAStream current;   // torch's, of that device
    void* stream = nullptr;
    Place(const at::Tensor& any, PyObject* s) : dev(any.device()), current(c10::cuda::getCurrentCUDAStream(dev.index())) {
        if (s == Py_None) stream = current.stream();
        else if (!stream_arg(s, &stream)) throw Raised();
    }
    at::Tensor make(c10::IntArrayRef shape, at::ScalarType type) const { return memory_on(stream, current, shape, type, true); }
    // memory of this call alone, given back when it returns
    at::Tensor scratch(c10::IntArrayRef shape, at::ScalarType type) const { return memory_on(stream, current, shape, type, false); }
};

const at::Tensor& need(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: expected a tensor, got %s", name, Py_TYPE(o)->tp_name);
        throw Raised();
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda()) throw Refused(name, "not on a GPU");
    if (!t.is_contiguous()) {
        PyErr_SetString(PyExc_AssertionError, "tensor is not contiguous");
        throw Raised();
    }
    return t;
}
void hold(const at::Tensor& t, const char* name, const c10::Device& dev, at::ScalarType type, c10::IntArrayRef shape) {
    if (t.device() != dev) throw Refused(name, "on another device");
    if (t.scalar_type() != type) throw Refused(name, "of another type than the call takes");
    if (t.sizes() != shape) throw Refused(name, "of another shape than the other tensors ask for");
}
// A tensor of this type and shape, or None.
void* maybe(PyObject* o, const char* name, const c10::Device& dev, at::ScalarType type, c10::IntArrayRef shape) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = need(o, name);
    hold(t, name, dev, type, shape);
    return t.data_ptr();
}
// An output: a tensor, or None / True = a new one, or (where the caller may do without) False.
struct Output {
    at::Tensor made;
    PyObject* given = nullptr;
    void* ptr = nullptr;
    Output(PyObject* o, const char* name, const Place& at, at::ScalarType type, c10::IntArrayRef shape, bool none_is_new) {
        if (o == Py_False || (o == Py_None && !none_is_new)) return;
        if (o == Py_None || o == Py_True) {
            made = at.make(shape, type);
            ptr = made.data_ptr();
        } else {
            ptr = maybe(o, name, at.dev, type, shape);
            given = o;
        }
    }
    PyObject* result() {
        if (given) return Py_NewRef(given);
        if (made.defined()) return THPVariable_Wrap(std::move(made));
        Py_RETURN_NONE;
    }
};
int32_t narrow(int64_t v, const char* name) {
    if (v > INT32_MAX) throw Refused(name, "too large");
    return (int32_t)v;
}

int64_t number(PyObject* o) {
    long long v;
    if (!int_arg(o, &v)) throw Raised();
    return v;
}

// route(logits, topk, renormalize, topk_idx, topk_w, stream): (topk_idx, topk_w), or the code
PyObject* py_route(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 6)) return nullptr;
        const at::Tensor& logits = need(a[0], "logits");
        if (logits.dim() != 2) throw Refused("logits", "not [tokens, experts]");
        const bool f32 = logits.scalar_type() == at::kFloat;
        if (!f32 && logits.scalar_type() != at::kBFloat16) throw Refused("logits", "neither fp32 nor bf16");
        const Place at(logits, a[5]);
        const int64_t T = logits.size(0), k = number(a[1]);
        if (k < 1 || k > 32) return PyLong_FromLong(UBEP_ERR_ARG);
        const int renorm = PyObject_IsTrue(a[2]);
        if (renorm < 0) return nullptr;
        Output idx(a[3], "topk_idx", at, at::kInt, {T, k}, true), w(a[4], "topk_w", at, at::kFloat, {T, k}, true);
        const void* pl = logits.data_ptr();
        const int32_t Ti = narrow(T, "logits"), E = narrow(logits.size(1), "logits");
        const int rc = without_gil([&] {
            return f_route(pl, f32 ? UBEP_LOGITS_F32 : UBEP_LOGITS_BF16, Ti, E, (int32_t)k, renorm, static_cast<int32_t*>(idx.ptr),
                           static_cast<float*>(w.ptr), at.dev.index(), at.stream);
        });
        if (rc != UBEP_OK) return PyLong_FromLong(rc);
        return Py_BuildValue("(NN)", idx.result(), w.result());
    } catch (...) {
        return refused_or_raised();
    }
}

// route_backward(logits, topk_idx, grad_w, renormalize, grad_logits, stream): grad_logits, or the code
PyObject* py_route_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 6)) return nullptr;
        const at::Tensor& logits = need(a[0], "logits");
        if (logits.dim() != 2) throw Refused("logits", "not [tokens, experts]");
        const bool f32 = logits.scalar_type() == at::kFloat;
        if (!f32 && logits.scalar_type() != at::kBFloat16) throw Refused("logits", "neither fp32 nor bf16");
        const Place at(logits, a[5]);
        const at::Tensor& idx = need(a[1], "topk_idx");
        if (idx.dim() != 2) throw Refused("topk_idx", "not [tokens, k]");
        const int64_t T = logits.size(0), k = idx.size(1);
        hold(idx, "topk_idx", at.dev, at::kInt, {T, k});
        const at::Tensor& gw = need(a[2], "grad_w");
        hold(gw, "grad_w", at.dev, at::kFloat, {T, k});
        const int renorm = PyObject_IsTrue(a[3]);
        if (renorm < 0) return nullptr;
        Output out(a[4], "grad_logits", at, logits.scalar_type(), logits.sizes(), true);
        const void* pl = logits.data_ptr();
        const int32_t *pi = idx.data_ptr<int32_t>(), Ti = narrow(T, "logits"), E = narrow(logits.size(1), "logits");
        const float* pg = gw.data_ptr<float>();
        const int rc = without_gil([&] {
            return f_route_backward(pl, f32 ? UBEP_LOGITS_F32 : UBEP_LOGITS_BF16, pi, pg, Ti, E, (int32_t)k, renorm, out.ptr, at.dev.index(),
                                    at.stream);
        });
        if (rc != UBEP_OK) return PyLong_FromLong(rc);
        return out.result();
    } catch (...) {
        return refused_or_raised();
    }
}

// The first three arguments of the expert calls: offset, count, status or None; the regions are those of `x`.
ubep_expert_rows_t rows_arg(PyObject* const* a, const Place& at, int64_t ranks, int64_t cap) {
    const at::Tensor &offset = need(a[0], "offset"), &count = need(a[1], "count");
    if (offset.dim() != 1) throw Refused("offset", "not [experts]");
    hold(offset, "offset", at.dev, at::kInt, {offset.size(0)});
    hold(count, "count", at.dev, at::kInt, {offset.size(0)});
    ubep_expert_rows_t r{};
    r.offset = offset.data_ptr<int32_t>();
    r.count = count.data_ptr<int32_t>();
    r.num_experts = narrow(offset.size(0), "offset");
    r.num_ranks = narrow(ranks, "x");
    r.rows_per_rank_cap = narrow(cap, "x");
    r.device = at.dev.index();
    r.status = static_cast<int32_t*>(maybe(a[2], "status", at.dev, at::kInt, {1}));
    return r;
}

// Rows with their scales or without: [ranks, cap, width].
struct RowsIn {
    const at::Tensor& t;
    int64_t R, cap, width;
    void* scale = nullptr;
    RowsIn(PyObject* x, PyObject* x_scale) : t(need(x, "x")) {
        if (t.dim() != 3) throw Refused("x", "not [ranks, rows, width]");
        R = t.size(0), cap = t.size(1), width = t.size(2);
        const auto type = t.scalar_type();
        if (x_scale != Py_None) {
            if (type != at::kFloat8_e4m3fn && type != at::kByte) throw Refused("x", "rows with scales are e4m3");
            if (width % 128 != 0) throw Refused("x", "rows with scales have a multiple of 128 channels");
            scale = maybe(x_scale, "x_scale", t.device(), at::kFloat, {R, cap, width / 128});
        } else if (type == at::kByte) {   // a receive region as the buffer's view shows it
            if (width % 2 != 0) throw Refused("x", "rows of bf16 have an even number of bytes");
            width /= 2;
        } else if (type != at::kBFloat16) {
            throw Refused("x", "neither bf16 rows nor e4m3 rows with scales");
        }
    }
};

// expert_gated(offset, count, status, x, x_scale, w, act, out, pre, stream): out, or the code
PyObject* py_gated(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 10)) return nullptr;
        const RowsIn x(a[3], a[4]);
        const Place at(x.t, a[9]);
        const ubep_expert_rows_t r = rows_arg(a, at, x.R, x.cap);
        const at::Tensor& w = need(a[5], "w");
        if (w.dim() != 4) throw Refused("w", "not [experts, 2, inner, width]");
        const int64_t I = w.size(2);
        hold(w, "w", at.dev, at::kBFloat16, {(int64_t)r.num_experts, 2, I, x.width});
        const int act = (int)number(a[6]);
        Output out(a[7], "out", at, at::kBFloat16, {x.R, x.cap, I}, true);
        void* pre = maybe(a[8], "pre", at.dev, at::kBFloat16, {x.R, x.cap, 2, I});
        at::Tensor scratch;
        if (x.scale) scratch = at.scratch({x.R, x.cap, x.width}, at::kBFloat16);
        const void *px = x.t.data_ptr(), *pw = w.data_ptr();
        void* ps = x.scale ? scratch.data_ptr() : nullptr;
        const int32_t H = narrow(x.width, "x"), Ii = narrow(I, "w");
        const int rc = without_gil([&] { return f_gated(&r, px, static_cast<const float*>(x.scale), pw, H, Ii, act, out.ptr, pre, ps, at.stream); });
        if (rc != UBEP_OK) return PyLong_FromLong(rc);
        return out.result();
    } catch (...) {
        return refused_or_raised();
    }
}

// expert_gated_backward(offset, count, status, x, x_scale, w, pre, grad_h, act, grad_pre, grad_x, grad_w, stream): (grad_x, grad_w), or the code
PyObject* py_gated_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 13)) return nullptr;
        const RowsIn x(a[3], a[4]);
        const Place at(x.t, a[12]);
        const ubep_expert_rows_t r = rows_arg(a, at, x.R, x.cap);
        const at::Tensor& w = need(a[5], "w");
        if (w.dim() != 4) throw Refused("w", "not [experts, 2, inner, width]");
        const int64_t I = w.size(2);
        hold(w, "w", at.dev, at::kBFloat16, {(int64_t)r.num_experts, 2, I, x.width});
        const at::Tensor &pre = need(a[6], "pre"), &gh = need(a[7], "grad_h");
        hold(pre, "pre", at.dev, at::kBFloat16, {x.R, x.cap, 2, I});
        hold(gh, "grad_h", at.dev, at::kBFloat16, {x.R, x.cap, I});
        const int act = (int)number(a[8]);
        at::Tensor room, scratch;
        void* gp = maybe(a[9], "grad_pre", at.dev, at::kBFloat16, {x.R, x.cap, 2, I});
        if (!gp) {
            room = at.scratch({x.R, x.cap, 2, I}, at::kBFloat16);
            gp = room.data_ptr();
        }
        Output gx(a[10], "grad_x", at, at::kBFloat16, {x.R, x.cap, x.width}, true), gw(a[11], "grad_w", at, at::kBFloat16, w.sizes(), true);
        if (x.scale && gw.ptr) scratch = at.scratch({2, x.R, x.cap, x.width}, at::kBFloat16);
        const void *px = x.t.data_ptr(), *pw = w.data_ptr(), *pp = pre.data_ptr(), *ph = gh.data_ptr();
        void* ps = scratch.defined() ? scratch.data_ptr() : nullptr;
        const int32_t H = narrow(x.width, "x"), Ii = narrow(I, "w");
        const int rc = without_gil([&] {
            return f_gated_backward(&r, px, static_cast<const float*>(x.scale), pw, pp, ph, H, Ii, act, gp, gx.ptr, gw.ptr, ps, at.stream);
        });
        if (rc != UBEP_OK) return PyLong_FromLong(rc);
        return Py_BuildValue("(NN)", gx.result(), gw.result());
    } catch (...) {
        return refused_or_raised();
    }
}

// expert_linear(offset, count, status, x, w, bias, row_scale, residual, act, out, pre, stream): out, or the code
PyObject* py_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 12)) return nullptr;
        const RowsIn x(a[3], Py_None);
        const Place at(x.t, a[11]);
        const ubep_expert_rows_t r = rows_arg(a, at, x.R, x.cap);
        const at::Tensor& w = need(a[4], "w");
        if (w.dim() != 3) throw Refused("w", "not [experts, out, in]");
        const int64_t N = w.size(1);
        hold(w, "w", at.dev, at::kBFloat16, {(int64_t)r.num_experts, N, x.width});
        const void* bias = maybe(a[5], "bias", at.dev, at::kBFloat16, {(int64_t)r.num_experts, N});
        const float* scale = static_cast<const float*>(maybe(a[6], "row_scale", at.dev, at::kFloat, {x.R, x.cap}));
        const void* residual = maybe(a[7], "residual", at.dev, at::kBFloat16, {x.R, x.cap, N});
        const int act = (int)number(a[8]);
        Output out(a[9], "out", at, at::kBFloat16, {x.R, x.cap, N}, true);
        void* pre = maybe(a[10], "pre", at.dev, at::kBFloat16, {x.R, x.cap, N});
        const void *px = x.t.data_ptr(), *pw = w.data_ptr();
        const int32_t K = narrow(x.width, "x"), Ni = narrow(N, "w");
        const int rc = without_gil([&] { return f_linear(&r, px, pw, bias, scale, residual, K, Ni, act, out.ptr, pre, at.stream); });
        if (rc != UBEP_OK) return PyLong_FromLong(rc);
        return out.result();
    } catch (...) {
        return refused_or_raised();
    }
}

// expert_linear_backward(offset, count, status, x, w, grad_y, pre, row_scale, act, grad_pre, grad_x, grad_w, grad_bias, grad_row_scale,
// stream): (grad_x, grad_w, grad_bias, grad_row_scale), or the code
PyObject* py_linear_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        if (!want_args(n, 15)) return nullptr;
        const RowsIn x(a[3], Py_None);
        const Place at(x.t, a[14]);
        const ubep_expert_rows_t r = rows_arg(a, at, x.R, x.cap);
        const at::Tensor& w = need(a[4], "w");
        if (w.dim() != 3) throw Refused("w", "not [experts, out, in]");
        const int64_t N = w.size(1);
        hold(w, "w", at.dev, at::kBFloat16, {(int64_t)r.num_experts, N, x.width});
        const at::Tensor& gy = need(a[5], "grad_y");
        hold(gy, "grad_y", at.dev, at::kBFloat16, {x.R, x.cap, N});
        const void* pre = maybe(a[6], "pre", at.dev, at::kBFloat16, {x.R, x.cap, N});
        const float* scale = static_cast<const float*>(maybe(a[7], "row_scale", at.dev, at::kFloat, {x.R, x.cap}));
        const int act = (int)number(a[8]);
        at::Tensor room;
        void* gp = maybe(a[9], "grad_pre", at.dev, at::kBFloat16, {x.R, x.cap, N});
        if (!gp && (act != UBEP_ACT_NONE || scale)) {
            room = at.scratch({x.R, x.cap, N}, at::kBFloat16);
            gp = room.data_ptr();
        }
        Output gx(a[10], "grad_x", at, at::kBFloat16, {x.R, x.cap, x.width}, true), gw(a[11], "grad_w", at, at::kBFloat16, w.sizes(), true),
            gb(a[12], "grad_bias", at, at::kBFloat16, {(int64_t)r.num_experts, N}, false),
            gs(a[13], "grad_row_scale", at, at::kFloat, {x.R, x.cap}, false);
        at::Tensor sums;
        if (gb.ptr) sums = at.scratch({std::max<int64_t>(r.num_experts, UBEP_EXPERT_PARTIALS), N}, at::kFloat);
        float* ps = gb.ptr ? sums.data_ptr<float>() : nullptr;
        const void *px = x.t.data_ptr(), *pw = w.data_ptr(), *py = gy.data_ptr();
        const int32_t K = narrow(x.width, "x"), Ni = narrow(N, "w");
        const int rc = without_gil([&] {
            return f_linear_backward(&r, px, pw, pre, scale, py, K, Ni, act, gp, gx.ptr, gw.ptr, gb.ptr, static_cast<float*>(gs.ptr), ps, at.stream);
        });
        if (rc != UBEP_OK) return PyLong_FromLong(rc);
        return Py_BuildValue("(NNNN)", gx.result(), gw.result(), gb.result(), gs.result());
    } catch (...) {
        return refused_or_raised();
    }
}

// current_stream(): the handle of torch's current stream
PyObject* py_current_stream(PyObject*, PyObject*) {
    try {
        return PyLong_FromVoidPtr(c10::cuda::getCurrentCUDAStream().stream());
    } catch (...) {
        return translate_exception();
    }
}

// bind(dispatch, combine, get_dispatch_layout, dispatch_sync, route, route_backward, expert_gated, expert_gated_backward, expert_linear,
// expert_linear_backward): addresses of the library's entry points
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void** const to[] = {reinterpret_cast<void**>(&f_dispatch),       reinterpret_cast<void**>(&f_combine),
                         reinterpret_cast<void**>(&f_layout),         reinterpret_cast<void**>(&f_dispatch_sync),
                         reinterpret_cast<void**>(&f_route),          reinterpret_cast<void**>(&f_route_backward),
                         reinterpret_cast<void**>(&f_gated),          reinterpret_cast<void**>(&f_gated_backward),
                         reinterpret_cast<void**>(&f_linear),         reinterpret_cast<void**>(&f_linear_backward)};
    if (!want_args(n, 10)) return nullptr;
    for (int i = 0; i < 10; ++i) {
        *to[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    Py_RETURN_NONE;
}

#define UBEP_FAST(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {
    UBEP_FAST("dispatch", py_dispatch),
    UBEP_FAST("dispatch_sync", py_dispatch_sync),
    UBEP_FAST("combine", py_combine),
    UBEP_FAST("combine_new", py_combine_new),
    UBEP_FAST("layout", py_layout),
    UBEP_FAST("layout_new", py_layout_new),
    UBEP_FAST("route", py_route),
    UBEP_FAST("route_backward", py_route_backward),
    UBEP_FAST("expert_gated", py_gated),
    UBEP_FAST("expert_gated_backward", py_gated_backward),
    UBEP_FAST("expert_linear", py_linear),
    UBEP_FAST("expert_linear_backward", py_linear_backward),
    UBEP_FAST("bind", py_bind),
    {"current_stream", py_current_stream, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) { return PyModule_Create(&kModule); }

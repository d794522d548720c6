// The calls of binding.py that enqueue work on device tensors, as a Python extension module: argument marshalling only.
//
// Why native.  A decode-sized call is ~20 us of GPU time behind three launches; through ctypes its host side took 24 us
// (stream lookup 3.4, three output tensors 7, argument conversion 4, the C call 8.5), which then was what a caller waited
// for.  Here the marshalling is ~1 us and the outputs ~1 us each.
//
// The module does not link the library: bind() is given the addresses of its functions, so that whichever build of it
// binding.py has loaded is the one called.  The GIL is released around every call, as ctypes does.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <optional>
#include <stdint.h>

#include "../../include/more_route.h"

namespace {

decltype(&more_route_ex) g_route_ex;
decltype(&more_route_psum) g_psum;
decltype(&more_dispatch) g_dispatch;
decltype(&more_route_full) g_full;
decltype(&more_merge_shards) g_merge;
decltype(&more_experts) g_experts;
decltype(&more_experts_workspace) g_experts_workspace;
decltype(&more_experts_path) g_experts_path;
decltype(&more_experts_backward) g_experts_backward;
decltype(&more_combine) g_combine;
decltype(&more_combine_backward) g_combine_backward;
decltype(&more_combine_workspace) g_combine_workspace;

struct Error {};                    // a Python exception is set

const at::Tensor& tensor(PyObject* o)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "expected a tensor, got %s", Py_TYPE(o)->tp_name);
        throw Error();
    }
    return THPVariable_Unpack(o);
}
void* ptr(PyObject* o) { return o == Py_None ? nullptr : const_cast<void*>(tensor(o).const_data_ptr()); }

int integer(PyObject* o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Error();
    if (v < INT32_MIN || v > INT32_MAX) {
        PyErr_SetString(PyExc_OverflowError, "argument does not fit in 32 bits");
        throw Error();
    }
    return (int)v;
}
int size(const at::Tensor& t, int dims, int d)
{
    if (t.dim() != dims) {
        PyErr_Format(PyExc_ValueError, "expected a tensor of %d dimensions, got %d", dims, (int)t.dim());
        throw Error();
    }
    return (int)t.size(d);
}
// None: torch's current stream of the current device
void* stream(PyObject* o)
{
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject* v = PyObject_GetAttrString(o, "cuda_stream");
    if (!v) throw Error();
    void* s = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    if (!s && PyErr_Occurred()) throw Error();
    return s;
}
void expect(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
        throw Error();
    }
}

template <class F>
PyObject* guarded(F body)
{
    HANDLE_TH_ERRORS
    try {
        return body();
    } catch (const Error&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

template <class F>
int released(F call)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}

int route_ex(PyObject* const* a, int k, int mode, void* idx, void* gate, void* counts, void* topval, void* lse, int path, int msplit,
             void* st)
{
    const at::Tensor &X = tensor(a[0]), &R2 = tensor(a[2]);
    void* r1 = ptr(a[1]);
    const int T = size(X, 2, 0), h = size(X, 2, 1), r = size(R2, 2, 0), M = size(R2, 2, 1);
    const void *x = X.const_data_ptr(), *r2 = R2.const_data_ptr();
    return released([&] {
        return g_route_ex(x, r1, r2, T, h, r, M, k, mode, static_cast<int32_t*>(idx), static_cast<float*>(gate),
                          static_cast<int32_t*>(counts), static_cast<float*>(topval), static_cast<float*>(lse), path, msplit, st);
    });
}

// bind(route_ex, psum, dispatch, full, merge, experts, experts_workspace, experts_path, experts_backward, combine,
// combine_backward, combine_workspace): addresses of the library's functions
PyObject* py_bind(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        constexpr int kFunctions = 12;
        expect(n, kFunctions);
        void* f[kFunctions];
        for (int i = 0; i < kFunctions; ++i)
            if (!(f[i] = PyLong_AsVoidPtr(a[i]))) {
                if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null function address");
                throw Error();
            }
        g_route_ex = reinterpret_cast<decltype(g_route_ex)>(f[0]);
        g_psum = reinterpret_cast<decltype(g_psum)>(f[1]);
        g_dispatch = reinterpret_cast<decltype(g_dispatch)>(f[2]);
        g_full = reinterpret_cast<decltype(g_full)>(f[3]);
        g_merge = reinterpret_cast<decltype(g_merge)>(f[4]);
        g_experts = reinterpret_cast<decltype(g_experts)>(f[5]);
        g_experts_workspace = reinterpret_cast<decltype(g_experts_workspace)>(f[6]);
        g_experts_path = reinterpret_cast<decltype(g_experts_path)>(f[7]);
        g_experts_backward = reinterpret_cast<decltype(g_experts_backward)>(f[8]);
        g_combine = reinterpret_cast<decltype(g_combine)>(f[9]);
        g_combine_backward = reinterpret_cast<decltype(g_combine_backward)>(f[10]);
        g_combine_workspace = reinterpret_cast<decltype(g_combine_workspace)>(f[11]);
        Py_RETURN_NONE;
    });
}

// route_ex(X, R1, R2, k, gate_mode, idx, gate, counts, topval, lse, path, msplit, stream) -> rc
PyObject* py_route_ex(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        expect(n, 13);
        return PyLong_FromLong(route_ex(a, integer(a[3]), integer(a[4]), ptr(a[5]), ptr(a[6]), ptr(a[7]), ptr(a[8]), ptr(a[9]),
                                        integer(a[10]), integer(a[11]), stream(a[12])));
    });
}

// route(X, R1, R2, k, gate_mode, want_topval, want_lse, path, msplit, stream) -> (rc, idx, gate, counts, topval, lse)
PyObject* py_route(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        expect(n, 10);
        const at::Tensor &X = tensor(a[0]), &R2 = tensor(a[2]);
        const int64_t T = size(X, 2, 0), M = size(R2, 2, 1);
        const int k = integer(a[3]);
        const bool want_topval = PyObject_IsTrue(a[5]) == 1, want_lse = PyObject_IsTrue(a[6]) == 1;
        const auto f32 = at::TensorOptions().device(X.device()).dtype(at::kFloat), i32 = f32.dtype(at::kInt);
        at::Tensor idx = at::empty({T, k}, i32), gate = at::empty({T, k}, f32), counts = at::empty({M}, i32), topval, lse;
        if (want_topval) topval = at::empty({T, k}, f32);
        if (want_lse) lse = at::empty({T}, f32);
        const int rc = route_ex(a, k, integer(a[4]), idx.data_ptr(), gate.data_ptr(), counts.data_ptr(),
                                want_topval ? topval.data_ptr() : nullptr, want_lse ? lse.data_ptr() : nullptr, integer(a[7]),
                                integer(a[8]), stream(a[9]));
        // (an undefined tensor is wrapped as None)
        return Py_BuildValue("(iNNNNN)", rc, THPVariable_Wrap(idx), THPVariable_Wrap(gate), THPVariable_Wrap(counts),
                             THPVariable_Wrap(topval), THPVariable_Wrap(lse));
    });
}

// psum(X, R1, R2, lse, out, path, stream) -> rc
PyObject* py_psum(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        expect(n, 7);
        const at::Tensor &X = tensor(a[0]), &R2 = tensor(a[2]);
        const int T = size(X, 2, 0), h = size(X, 2, 1), r = size(R2, 2, 0), M = size(R2, 2, 1), path = integer(a[5]);
        void *r1 = ptr(a[1]), *lse = ptr(a[3]), *out = ptr(a[4]), *st = stream(a[6]);
        return PyLong_FromLong(released([&] {
            return g_psum(X.const_data_ptr(), r1, R2.const_data_ptr(), T, h, r, M, static_cast<const float*>(lse),
                          static_cast<float*>(out), path, st);
        }));
    });
}

// dispatch(idx, counts, offsets, pairs, stream) -> rc
PyObject* py_dispatch(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        expect(n, 5);
        const at::Tensor &idx = tensor(a[0]), &counts = tensor(a[1]);
        const int T = size(idx, 2, 0), k = size(idx, 2, 1), M = counts.dim() > 0 ? (int)counts.size(0) : size(counts, 1, 0);
        void *off = ptr(a[2]), *pairs = ptr(a[3]), *st = stream(a[4]);
        return PyLong_FromLong(released([&] {
            return g_dispatch(static_cast<const int32_t*>(idx.const_data_ptr()), static_cast<const int32_t*>(counts.const_data_ptr()), T,
                              k, M, static_cast<int32_t*>(off), static_cast<int32_t*>(pairs), st);
        }));
    });
}

// full(X, W, k, gate_mode, idx, gate, counts, topval, lse, msplit, stream) -> rc
PyObject* py_full(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        expect(n, 11);
        const at::Tensor &X = tensor(a[0]), &Wt = tensor(a[1]);
        const int T = size(X, 2, 0), h = size(X, 2, 1), M = size(Wt, 2, 1), k = integer(a[2]), mode = integer(a[3]);
        void *idx = ptr(a[4]), *gate = ptr(a[5]), *counts = ptr(a[6]), *topval = ptr(a[7]), *lse = ptr(a[8]);
        const int msplit = integer(a[9]);
        void* st = stream(a[10]);
        return PyLong_FromLong(released([&] {
            return g_full(X.const_data_ptr(), Wt.const_data_ptr(), T, h, M, k, mode, static_cast<int32_t*>(idx), static_cast<float*>(gate),
                          static_cast<int32_t*>(counts), static_cast<float*>(topval), static_cast<float*>(lse), msplit, st);
        }));
    });
}

// merge(idx, topval, lse, shard_base, M, gate_mode, out_idx, out_gate, counts, out_topval, out_lse, stream) -> rc
PyObject* py_merge(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        expect(n, 12);
        const at::Tensor& idx = tensor(a[0]);
        const int S = size(idx, 3, 0), T = size(idx, 3, 1), k = size(idx, 3, 2);
        int32_t base[MORE_MERGE_MAX_SHARDS];
        const bool based = a[3] != Py_None;
        if (based && S <= MORE_MERGE_MAX_SHARDS) {           // (more shards than that: the library refuses the call)
            PyObject* seq = PySequence_Fast(a[3], "shard_base is a sequence of integers");
            if (!seq) throw Error();
            const Py_ssize_t count = PySequence_Fast_GET_SIZE(seq);
            if (count != S) {
                Py_DECREF(seq);
                PyErr_Format(PyExc_IndexError, "shard_base has %zd entries for %d shards", count, S);
                throw Error();
            }
            for (int s = 0; s < S; ++s) {
                PyObject* v = PyNumber_Long(PySequence_Fast_GET_ITEM(seq, s));
                const long b = v ? PyLong_AsLong(v) : -1;
                Py_XDECREF(v);
                if (b == -1 && PyErr_Occurred()) {
                    Py_DECREF(seq);
                    throw Error();
                }
                base[s] = (int32_t)b;
            }
            Py_DECREF(seq);
        }
        const int M = integer(a[4]), mode = integer(a[5]);
        void *val = ptr(a[1]), *lse = ptr(a[2]), *oi = ptr(a[6]), *og = ptr(a[7]), *oc = ptr(a[8]), *ov = ptr(a[9]), *ol = ptr(a[10]);
        void* st = stream(a[11]);
        return PyLong_FromLong(released([&] {
            return g_merge(static_cast<const int32_t*>(idx.const_data_ptr()), static_cast<const float*>(val), static_cast<const float*>(lse),
                           based ? base : nullptr, S, T, k, M, mode, static_cast<int32_t*>(oi), static_cast<float*>(og),
                           static_cast<float*>(ov), static_cast<float*>(ol), static_cast<int32_t*>(oc), st);
        }));
    });
}

// ------------------------------------------------------------------------------------------------ experts, combine
// These calls check their tensors (type, shape, contiguity, device) before the library sees pointers.

[[noreturn]] void refuse(const char* name, const char* why)
{
    PyErr_Format(PyExc_ValueError, "%s: %s", name, why);
    throw Error();
}

// A contiguous tensor of that type and shape on the current device; None gives nullptr where it may.
void* checked(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> shape, bool optional = false)
{
    if (o == Py_None && optional) return nullptr;
    const at::Tensor& t = tensor(o);
    if (!t.is_cuda()) refuse(name, "expected a CUDA tensor");
    if (t.get_device() != c10::cuda::current_device()) refuse(name, "is not on the current device");
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_TypeError, "%s: expected %s, got %s", name, c10::toString(type), c10::toString(t.scalar_type()));
        throw Error();
    }
    if (t.sizes() != c10::IntArrayRef(shape.begin(), shape.size())) refuse(name, "has another shape than the other arguments ask for");
    if (!t.is_contiguous()) refuse(name, "is not contiguous");
    return const_cast<void*>(t.const_data_ptr());
}
int64_t extent(PyObject* o, const char* name, int dims, int d)
{
    const at::Tensor& t = tensor(o);
    if (t.dim() != dims) {
        PyErr_Format(PyExc_ValueError, "%s: expected %d dimensions, got %d", name, dims, (int)t.dim());
        throw Error();
    }
    if (t.size(d) > INT32_MAX) refuse(name, "a dimension does not fit in 32 bits");
    return t.size(d);
}

// What a call allocates belongs to the stream that it runs on.
struct OnStream {
    void* st;
    std::optional<c10::cuda::CUDAStreamGuard> guard;
    explicit OnStream(PyObject* o) : st(stream(o))
    {
        if (o != Py_None) guard.emplace(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(st), c10::cuda::current_device()));
    }
};
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type)
{
    return at::empty(shape, at::TensorOptions().device(at::Device(at::kCUDA, c10::cuda::current_device())).dtype(type));
}
// The caller's workspace, or one of `bytes` of torch's memory, kept alive by `own` until the call returns (the memory is then only
// given to work behind this call's on its stream).
void* workspace(PyObject* o, int64_t bytes, at::Tensor& own, int64_t* have)
{
    if (o != Py_None) {
        const at::Tensor& t = tensor(o);
        *have = (int64_t)t.nbytes();
        return checked(o, "workspace", at::kByte, {*have});
    }
    *have = bytes;
    if (bytes <= 0) return nullptr;
    own = fresh({bytes}, at::kByte);
    return own.data_ptr();
}

struct ExpertsSizes {
    int64_t T, h, s, M, k;
    ExpertsSizes(PyObject* X, PyObject* W2, PyObject* idx)
        : T(extent(X, "X", 2, 0)), h(extent(X, "X", 2, 1)), s(extent(W2, "W2", 3, 1)), M(extent(W2, "W2", 3, 0)), k(extent(idx, "idx", 2, 1))
    {
    }
};

// The given output, or a fresh one where it may be made; nullptr where it is neither.
struct Output {
    at::Tensor made;
    PyObject* given;
    void* at;
    Output(PyObject* o, const char* name, at::ScalarType type, std::initializer_list<int64_t> shape, bool make) : given(o), at(nullptr)
    {
        if (o != Py_None) at = checked(o, name, type, shape);
        else if (make) {
            made = fresh(at::IntArrayRef(shape.begin(), shape.size()), type);
            at = made.data_ptr();
        }
    }
    PyObject* result()            // a new reference
    {
        if (given != Py_None) {
            Py_INCREF(given);
            return given;
        }
        return THPVariable_Wrap(made);
    }
};

// experts(X, W1, W2, idx, offsets, pairs, y, hidden, make_hidden, path, workspace, stream) -> (rc, y, hidden)
PyObject* py_experts(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        expect(n, 12);
        const ExpertsSizes z(a[0], a[2], a[3]);
        void *x = checked(a[0], "X", at::kBFloat16, {z.T, z.h}), *w1 = checked(a[1], "W1", at::kBFloat16, {z.M, z.h, 2 * z.s}),
             *w2 = checked(a[2], "W2", at::kBFloat16, {z.M, z.s, z.h}), *idx = checked(a[3], "idx", at::kInt, {z.T, z.k}),
             *off = checked(a[4], "offsets", at::kInt, {z.M + 1}, true), *pairs = checked(a[5], "pairs", at::kInt, {z.T * z.k}, true);
        const OnStream on(a[11]);
        const int path = integer(a[9]);
        const int T = (int)z.T, h = (int)z.h, s = (int)z.s, M = (int)z.M, k = (int)z.k;
        Output y(a[6], "out_y", at::kBFloat16, {z.T * z.k, z.h}, true);
        Output hidden(a[7], "out_hidden", at::kBFloat16, {z.T * z.k, 2 * z.s}, PyObject_IsTrue(a[8]) == 1);
        at::Tensor own;
        int64_t have = 0;
        void* ws = nullptr;
        const bool tiles = path == MORE_EXPERTS_TILES || (path == MORE_EXPERTS_AUTO && off && pairs && (hidden.at || g_experts_path(T, h, s, M, k) == MORE_EXPERTS_TILES));
        if (tiles || a[10] != Py_None) ws = workspace(a[10], g_experts_workspace(T, h, s, M, k, 0), own, &have);
        const int rc = released([&] {
            return g_experts(x, w1, w2, static_cast<const int32_t*>(idx), static_cast<const int32_t*>(off), static_cast<const int32_t*>(pairs), T, h,
                             s, M, k, y.at, hidden.at, path, ws, have, on.st);
        });
        return Py_BuildValue("(iNN)", rc, y.result(), hidden.result());
    });
}

// experts_backward(X, W1, W2, idx, offsets, pairs, gate, hidden, dout, dx, dgate, dw1, dw2, make, workspace, stream)
// -> (rc, dx, dgate, dw1, dw2); make: bits of the outputs to allocate where they are None
PyObject* py_experts_backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        expect(n, 16);
        const ExpertsSizes z(a[0], a[2], a[3]);
        void *x = checked(a[0], "X", at::kBFloat16, {z.T, z.h}), *w1 = checked(a[1], "W1", at::kBFloat16, {z.M, z.h, 2 * z.s}),
             *w2 = checked(a[2], "W2", at::kBFloat16, {z.M, z.s, z.h}), *idx = checked(a[3], "idx", at::kInt, {z.T, z.k}),
             *off = checked(a[4], "offsets", at::kInt, {z.M + 1}), *pairs = checked(a[5], "pairs", at::kInt, {z.T * z.k}),
             *gate = checked(a[6], "gate", at::kFloat, {z.T, z.k}), *hidden = checked(a[7], "hidden", at::kBFloat16, {z.T * z.k, 2 * z.s}),
             *dout = checked(a[8], "dout", at::kBFloat16, {z.T, z.h});
        const OnStream on(a[15]);
        const int make = integer(a[13]);
        const int T = (int)z.T, h = (int)z.h, s = (int)z.s, M = (int)z.M, k = (int)z.k;
        Output dx(a[9], "out_dx", at::kBFloat16, {z.T, z.h}, make & 1), dgate(a[10], "out_dgate", at::kFloat, {z.T, z.k}, make & 2),
            dw1(a[11], "out_dw1", at::kBFloat16, {z.M, z.h, 2 * z.s}, make & 4), dw2(a[12], "out_dw2", at::kBFloat16, {z.M, z.s, z.h}, make & 8);
        at::Tensor own;
        int64_t have = 0;
        void* ws = workspace(a[14], g_experts_workspace(T, h, s, M, k, 1), own, &have);
        const int rc = released([&] {
            return g_experts_backward(x, w1, w2, static_cast<const int32_t*>(idx), static_cast<const int32_t*>(off),
                                      static_cast<const int32_t*>(pairs), static_cast<const float*>(gate), hidden, dout, T, h, s, M, k, dx.at,
                                      static_cast<float*>(dgate.at), dw1.at, dw2.at, ws, have, on.st);
        });
        return Py_BuildValue("(iNNNN)", rc, dx.result(), dgate.result(), dw1.result(), dw2.result());
    });
}

double real(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Error();
    return v;
}
// bf16 or fp32
at::ScalarType residual_type(PyObject* o, const char* name)
{
    const at::ScalarType type = tensor(o).scalar_type();
    if (type != at::kBFloat16 && type != at::kFloat) {
        PyErr_Format(PyExc_TypeError, "%s: expected BFloat16 or Float, got %s", name, c10::toString(type));
        throw Error();
    }
    return type;
}

// combine(Y, gate, residual, w_post, scale, w_pre, eps, k, out_residual, out_x, out_sum, make, stream) -> (rc, residual, x, sum)
// k: slots per token where there is no gate (0: by the shapes); make: bits of the outputs to allocate where they are None
PyObject* py_combine(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        expect(n, 13);
        PyObject *Y = a[0], *gate = a[1], *res = a[2];
        int64_t T = 0, h = 0, k = integer(a[7]);
        if (Y == Py_None && res == Py_None) refuse("combine", "neither rows nor a residual");
        if (k < 0) refuse("k", "is negative");
        if (Y != Py_None) h = extent(Y, "Y", 2, 1);
        else h = extent(res, "residual", 2, 1);
        if (gate != Py_None) {
            T = extent(gate, "gate", 2, 0);
            k = extent(gate, "gate", 2, 1);
        } else if (res != Py_None) {
            T = extent(res, "residual", 2, 0);
            if (k == 0) k = Y != Py_None && T > 0 ? extent(Y, "Y", 2, 0) / T : 1;
        } else {
            if (k == 0) k = 1;
            T = extent(Y, "Y", 2, 0) / k;
        }
        // (without a residual its type is that of the output that is given, or bf16)
        const at::ScalarType type = res != Py_None ? residual_type(res, "residual") : (a[8] != Py_None ? residual_type(a[8], "out_residual") : at::kBFloat16);
        void *y = checked(Y, "Y", at::kBFloat16, {T * k, h}, true), *g = checked(gate, "gate", at::kFloat, {T, k}, true),
             *r = checked(res, "residual", type, {T, h}, true), *wp = checked(a[3], "w_post", at::kFloat, {h}, true),
             *sc = checked(a[4], "scale", at::kFloat, {h}, true), *wn = checked(a[5], "w_pre", at::kFloat, {h}, true);
        const double eps = real(a[6]);
        const OnStream on(a[12]);
        const int make = integer(a[11]);
        Output orr(a[8], "out_residual", type, {T, h}, make & 1), ox(a[9], "out_x", at::kBFloat16, {T, h}, make & 2),
            os(a[10], "out_sum", at::kBFloat16, {T, h}, make & 4);
        const int rc = released([&] {
            return g_combine(y, static_cast<const float*>(g), r, type == at::kFloat ? MORE_RESIDUAL_FP32 : MORE_RESIDUAL_BF16,
                             static_cast<const float*>(wp), static_cast<const float*>(sc), static_cast<const float*>(wn), (float)eps, (int)T, (int)h,
                             (int)k, orr.at, ox.at, os.at, on.st);
        });
        return Py_BuildValue("(iNNN)", rc, orr.result(), ox.result(), os.result());
    });
}

// combine_backward(dresidual, dx, sum, residual_out, w_post, scale, w_pre, eps, out_dresidual, out_dsum, out_dw_post, out_dscale,
// out_dw_pre, make, workspace, stream) -> (rc, dresidual, dsum, dw_post, dscale, dw_pre)
PyObject* py_combine_backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        expect(n, 16);
        PyObject* shape = a[0] != Py_None ? a[0] : a[1];
        if (shape == Py_None) refuse("combine_backward", "neither the residual's gradient nor that of x");
        const int64_t T = extent(shape, "gradient", 2, 0), h = extent(shape, "gradient", 2, 1);
        const at::ScalarType type = a[0] != Py_None ? residual_type(a[0], "dresidual")
                                    : a[3] != Py_None ? residual_type(a[3], "residual_out") : at::kBFloat16;
        void *dr = checked(a[0], "dresidual", type, {T, h}, true), *dx = checked(a[1], "dx", at::kBFloat16, {T, h}, true),
             *sum = checked(a[2], "sum", at::kBFloat16, {T, h}, true), *ro = checked(a[3], "residual_out", type, {T, h}, true),
             *wp = checked(a[4], "w_post", at::kFloat, {h}, true), *sc = checked(a[5], "scale", at::kFloat, {h}, true),
             *wn = checked(a[6], "w_pre", at::kFloat, {h}, true);
        const double eps = real(a[7]);
        const OnStream on(a[15]);
        const int make = integer(a[13]);
        Output odr(a[8], "out_dresidual", type, {T, h}, make & 1), ods(a[9], "out_dsum", at::kBFloat16, {T, h}, make & 2),
            owp(a[10], "out_dw_post", at::kFloat, {h}, make & 4), osc(a[11], "out_dscale", at::kFloat, {h}, make & 8),
            own_(a[12], "out_dw_pre", at::kFloat, {h}, make & 16);
        at::Tensor own;
        int64_t have = 0;
        void* ws = nullptr;
        if (owp.at || osc.at || own_.at) ws = workspace(a[14], g_combine_workspace((int)T, (int)h), own, &have);
        const int rc = released([&] {
            return g_combine_backward(dr, dx, sum, ro, type == at::kFloat ? MORE_RESIDUAL_FP32 : MORE_RESIDUAL_BF16, static_cast<const float*>(wp),
                                      static_cast<const float*>(sc), static_cast<const float*>(wn), (float)eps, (int)T, (int)h, odr.at, ods.at,
                                      static_cast<float*>(owp.at), static_cast<float*>(osc.at), static_cast<float*>(own_.at), ws, have, on.st);
        });
        return Py_BuildValue("(iNNNNN)", rc, odr.result(), ods.result(), owp.result(), osc.result(), own_.result());
    });
}

#define MORE_FAST(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    MORE_FAST("bind", py_bind), MORE_FAST("route", py_route), MORE_FAST("route_ex", py_route_ex), MORE_FAST("psum", py_psum),
    MORE_FAST("dispatch", py_dispatch), MORE_FAST("full", py_full), MORE_FAST("merge", py_merge),
    MORE_FAST("experts", py_experts), MORE_FAST("experts_backward", py_experts_backward), MORE_FAST("combine", py_combine),
    MORE_FAST("combine_backward", py_combine_backward), {nullptr, nullptr, 0, nullptr}};
// (the text by which build.py tells whether the module fits the torch and the Python that are installed)
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_more_binding", "built for " MORE_BUILT_FOR ";", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__more_binding() { return PyModule_Create(&module); }

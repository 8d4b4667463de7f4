// Argument marshalling of binding.py's hot entry points: torch tensors to device pointers, Python integers and the shape
// structure to the C ABI's arguments.  What ctypes takes for that is a third of a call's host time (us, a forward / backward
// step that launches nothing 1.65 / 2.24, here 0.41 / 0.44), and rings of short blocks last as long as their launches.
//
// Each does what the ctypes call of the same entry point does, with the same conversions: the
// library's function is handed over by its address, the interpreter's lock is given up during the call, and `stream` is
// a function that gives the stream's handle.
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>

#include "striped_attn.h"

namespace {

PyTypeObject* shape_type = nullptr;
PyObject* other_integer = nullptr;          // for what is no Python integer

struct ToStop {};          // a Python error is set

void* pointer(PyObject* o) {
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.is_cuda()) return t.data_ptr();
    }
    PyErr_SetString(PyExc_TypeError, "expected a GPU tensor");
    throw ToStop();
}
// as ctypes converts to c_int32 and c_int64: no floats, whatever has __index__, bits beyond are dropped
uint64_t integer(PyObject* o) {
    PyObject* other = nullptr;
    if (!PyIndex_Check(o)) {
        o = other = PyObject_CallOneArg(other_integer, o);
        if (!o) throw ToStop();
    }
    const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
    Py_XDECREF(other);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) throw ToStop();
    return v;
}
int32_t int32(PyObject* o) { return (int32_t)(uint32_t)integer(o); }
// A length that bounds others, for which the largest number that 32 bits hold says as much as any beyond it: the nearest one (of a window of 2^32 + 5
// the bits dropped would leave one of 5).
int32_t bound(PyObject* o) {
    PyObject* const whole = PyIndex_Check(o) ? PyNumber_Index(o) : PyObject_CallOneArg(other_integer, o);
    if (!whole) throw ToStop();
    int beyond = 0;
    const long long v = PyLong_AsLongLongAndOverflow(whole, &beyond);
    Py_DECREF(whole);
    if (beyond) return beyond > 0 ? INT32_MAX : INT32_MIN;
    return (int32_t)std::min<long long>(std::max<long long>(v, INT32_MIN), INT32_MAX);
}
// asked when the tensors have been looked at
void* stream(PyObject* ask) {
    PyObject* o = PyObject_CallNoArgs(ask);
    if (!o) throw ToStop();
    void* const st = reinterpret_cast<void*>((uintptr_t)PyLong_AsUnsignedLongLongMask(o));
    Py_DECREF(o);
    if (PyErr_Occurred()) throw ToStop();
    return st;
}
void* address(PyObject* o) { return reinterpret_cast<void*>((uintptr_t)integer(o)); }
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw ToStop();
    return (float)v;
}
struct Shape {
    Py_buffer b;
    explicit Shape(PyObject* o) {
        if (!shape_type || !PyObject_TypeCheck(o, shape_type)) {
            PyErr_SetString(PyExc_TypeError, "expected a SaShape");
            throw ToStop();
        }
        if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE)) throw ToStop();
    }
    ~Shape() { PyBuffer_Release(&b); }
    const void* at() const { return b.buf; }
};

template <typename F>
PyObject* run(F call) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}
template <typename F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F body) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
        return nullptr;
    }
    try {
        return body();
    } catch (const ToStop&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

using I = int32_t;
using P = void*;
using C = const void*;
#define ENTRY(name) PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n)

// (function address, 2 tensors, shape, stream)
ENTRY(two) {
    return guarded(n, 5, [&] {
        const auto f = reinterpret_cast<int (*)(P, P, C, P)>(address(a[0]));
        P t0 = pointer(a[1]), t1 = pointer(a[2]), st = stream(a[4]);
        const Shape s(a[3]);
        return run([&] { return f(t0, t1, s.at(), st); });
    });
}
// (function address, 3 tensors, shape, stream)
ENTRY(three) {
    return guarded(n, 6, [&] {
        const auto f = reinterpret_cast<int (*)(P, P, P, C, P)>(address(a[0]));
        P t0 = pointer(a[1]), t1 = pointer(a[2]), t2 = pointer(a[3]), st = stream(a[5]);
        const Shape s(a[4]);
        return run([&] { return f(t0, t1, t2, s.at(), st); });
    });
}
// (function address, q, k, v, o, lse, q_dev, kv_dev, N, layout, shape, stream)
ENTRY(step_fwd) {
    return guarded(n, 12, [&] {
        const auto f = reinterpret_cast<int (*)(P, P, P, P, P, I, I, I, I, C, P)>(address(a[0]));
        P t[5];
        for (int i = 0; i < 5; ++i) t[i] = pointer(a[1 + i]);
        const I q = int32(a[6]), kv = int32(a[7]), N = int32(a[8]), layout = int32(a[9]);
        P st = stream(a[11]);
        const Shape s(a[10]);
        return run([&] { return f(t[0], t[1], t[2], t[3], t[4], q, kv, N, layout, s.at(), st); });
    });
}
// (function address, q, k, v, dout, lse, delta, dq, dk, dv, q_dev, kv_dev, N, layout, shape, stream)
ENTRY(step_bwd) {
    return guarded(n, 16, [&] {
        const auto f = reinterpret_cast<int (*)(P, P, P, P, P, P, P, P, P, I, I, I, I, C, P)>(address(a[0]));
        P t[9];
        for (int i = 0; i < 9; ++i) t[i] = pointer(a[1 + i]);
        const I q = int32(a[10]), kv = int32(a[11]), N = int32(a[12]), layout = int32(a[13]);
        P st = stream(a[15]);
        const Shape s(a[14]);
        return run([&] { return f(t[0], t[1], t[2], t[3], t[4], t[5], t[6], t[7], t[8], q, kv, N, layout, s.at(), st); });
    });
}
// (function address, Q, K, V, O, LSE, N, layout, shape, q_dev_only, stream)
ENTRY(ring_fwd) {
    return guarded(n, 11, [&] {
        const auto f = reinterpret_cast<int (*)(P, P, P, P, P, I, I, C, I, P, P)>(address(a[0]));
        P t[5];
        for (int i = 0; i < 5; ++i) t[i] = pointer(a[1 + i]);
        const I N = int32(a[6]), layout = int32(a[7]), only = int32(a[9]);
        P st = stream(a[10]);
        const Shape s(a[8]);
        return run([&] { return f(t[0], t[1], t[2], t[3], t[4], N, layout, s.at(), only, nullptr, st); });
    });
}
// (function address, Q, K, V, dO, O, LSE, delta, dQ, dK, dV, N, layout, shape, q_dev_only, stream)
ENTRY(ring_bwd) {
    return guarded(n, 16, [&] {
        const auto f = reinterpret_cast<int (*)(P, P, P, P, P, P, P, P, P, P, I, I, C, I, P, P)>(address(a[0]));
        P t[10];
        for (int i = 0; i < 10; ++i) t[i] = pointer(a[1 + i]);
        const I N = int32(a[11]), layout = int32(a[12]), only = int32(a[14]);
        P st = stream(a[15]);
        const Shape s(a[13]);
        return run([&] {
            return f(t[0], t[1], t[2], t[3], t[4], t[5], t[6], t[7], t[8], t[9], N, layout, s.at(), only, nullptr, st);
        });
    });
}
// (function address, x, y, pos, pos_stride_b, shape, base, inverse, stream)
ENTRY(rope) {
    return guarded(n, 9, [&] {
        const auto f = reinterpret_cast<int (*)(P, P, P, int64_t, C, float, I, P)>(address(a[0]));
        P x = pointer(a[1]), y = pointer(a[2]), pos = pointer(a[3]), st = stream(a[8]);
        const int64_t stride = (int64_t)integer(a[4]);
        const float base = real(a[6]);
        const I inverse = int32(a[7]);
        const Shape s(a[5]);
        return run([&] { return f(x, y, pos, stride, s.at(), base, inverse, st); });
    });
}
// What a permutation along axis o moves, rows of `inner` bytes: as an index of t's shape, from the end if negative
struct Extent { int64_t outer, rows, inner; };
Extent extent(const at::Tensor& t, PyObject* o) {
    const int64_t dims = t.dim(), axis = PyNumber_AsSsize_t(o, PyExc_IndexError);
    if (axis == -1 && PyErr_Occurred()) throw ToStop();
    if (axis < -dims || axis >= dims) {
        PyErr_SetString(PyExc_IndexError, "tuple index out of range");
        throw ToStop();
    }
    const int64_t at = axis < 0 ? axis + dims : axis;
    Extent e = {1, t.size(at), t.element_size()};
    for (int64_t i = 0; i < at; ++i) e.outer *= t.size(i);
    for (int64_t i = at + 1; i < dims; ++i) e.inner *= t.size(i);
    return e;
}
const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) pointer(Py_None);
    return THPVariable_Unpack(o);
}
// (tensor, axis): its extent
ENTRY(extent_of) {
    return guarded(n, 2, [&] {
        const Extent e = extent(tensor(a[0]), a[1]);
        return Py_BuildValue("LLL", (long long)e.outer, (long long)e.rows, (long long)e.inner);
    });
}
// (function address, src, dst, N, seq_axis, stream): the tensors' sizes are looked at here.  None: not contiguous with equal
// shape and type
ENTRY(permute) {
    return guarded(n, 6, [&]() -> PyObject* {
        const auto f = reinterpret_cast<int (*)(P, P, int64_t, int64_t, int64_t, I, P)>(address(a[0]));
        const at::Tensor &src = tensor(a[1]), &dst = tensor(a[2]);
        if (!src.is_contiguous() || !dst.is_contiguous() || src.sizes() != dst.sizes() || src.scalar_type() != dst.scalar_type())
            Py_RETURN_NONE;
        const I N = int32(a[3]);
        const Extent e = extent(src, a[4]);
        P s = pointer(a[1]), d = pointer(a[2]), st = stream(a[5]);
        return run([&] { return f(s, d, e.outer, e.rows, e.inner, N, st); });
    });
}
// ---- packed sequences and the paged cache: sizes and strides are read from the tensors here.  All tensors of a call lie on the
// current device, whose stream the call goes to.
[[noreturn]] void refuse(PyObject* error, const char* why) {
    PyErr_SetString(error, why);
    throw ToStop();
}
struct Call {
    int64_t device;
    explicit Call(PyObject* ask) {
        PyObject* o = PyObject_CallNoArgs(ask);
        if (!o) throw ToStop();
        device = PyLong_AsLongLong(o);
        Py_DECREF(o);
        if (device == -1 && PyErr_Occurred()) throw ToStop();
    }
    const at::Tensor& operator()(PyObject* o) const {
        const at::Tensor& t = tensor(o);
        if (!t.is_cuda()) pointer(Py_None);
        if (t.get_device() != device) refuse(PyExc_ValueError, "tensors must be on the current device");
        return t;
    }
    // rows of int32
    const at::Tensor& ids(PyObject* o, const char* why) const {
        const at::Tensor& t = (*this)(o);
        if (t.scalar_type() != at::kInt || !t.is_contiguous()) refuse(PyExc_TypeError, why);
        return t;
    }
};
int32_t type_of(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return SA_F32;
    if (t.scalar_type() == at::kBFloat16) return SA_BF16;
    refuse(PyExc_TypeError, "tensors must be float32 or bfloat16");
}
int32_t size(const at::Tensor& t, int64_t i) {
    if (t.size(i) > INT32_MAX) refuse(PyExc_ValueError, "a size is beyond 32 bits");
    return (int32_t)t.size(i);
}
// [rows, heads, d]: strides of rows and heads; of a single one whatever fits
struct Strides { int64_t s, h; };
Strides strides(const at::Tensor& t) {
    if (t.dim() != 3) refuse(PyExc_ValueError, "expected [rows, heads, d]");
    if (t.size(2) > 1 && t.stride(2) != 1) refuse(PyExc_ValueError, "the head dimension must be contiguous");
    const int64_t h = t.size(1) == 1 ? t.size(2) : t.stride(1);
    return {t.size(0) <= 1 ? h * t.size(1) : t.stride(0), h};
}
// as t but for what it holds
void same(const at::Tensor& t, const at::Tensor& as, const char* why) {
    if (t.sizes() != as.sizes() || t.scalar_type() != as.scalar_type()) refuse(PyExc_ValueError, why);
    for (int64_t i = 0; i < t.dim(); ++i)
        if (t.size(i) > 1 && t.stride(i) != as.stride(i)) refuse(PyExc_ValueError, why);
}
void statistics(const at::Tensor& t, int64_t n0, int64_t n1, const char* why) {
    if (t.scalar_type() != at::kFloat || t.dim() != 2 || t.size(0) != n0 || t.size(1) != n1 || (n1 > 1 && t.stride(1) != 1))
        refuse(PyExc_ValueError, why);
}
void* at_of(const at::Tensor& t) { return t.data_ptr(); }
const at::Tensor* maybe(const Call& on, PyObject* o) { return o == Py_None ? nullptr : &on(o); }
void* at_of(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
sa_packed packed_of(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& offsets, const at::Tensor& lse, PyObject* max_len,
                    PyObject* scale) {
    const Strides qs = strides(q), ks = strides(k);
    same(v, k, "k and v must have the same shape, type and strides");
    if (k.size(0) != q.size(0) || k.size(2) != q.size(2) || k.scalar_type() != q.scalar_type())
        refuse(PyExc_ValueError, "q and k must have the same rows, head dimension and type");
    if (offsets.dim() != 1 || offsets.size(0) < 1) refuse(PyExc_ValueError, "offsets must hold one more number than there are sequences");
    statistics(lse, q.size(1), q.size(0), "lse must be float32 [heads, rows], rows contiguous");
    return {size(offsets, 0) - 1, size(q, 0), bound(max_len), size(q, 1), size(k, 1), size(q, 2), qs.h, qs.s, ks.h, ks.s,
            q.size(1) == 1 ? q.size(0) : lse.stride(0), type_of(q), real(scale)};
}
const char* const OFFSETS = "offsets must be a contiguous int32 tensor";
// (function address, q, k, v, offsets, out, lse, max_len, scale, device, stream)
ENTRY(packed_fwd) {
    return guarded(n, 11, [&] {
        const auto f = reinterpret_cast<decltype(&sa_attn_packed_fwd)>(address(a[0]));
        const Call on(a[9]);
        const at::Tensor &q = on(a[1]), &k = on(a[2]), &v = on(a[3]), &off = on.ids(a[4], OFFSETS), &out = on(a[5]), &lse = on(a[6]);
        const sa_packed s = packed_of(q, k, v, off, lse, a[7], a[8]);
        same(out, q, "out must have q's shape, type and strides");
        void* st = stream(a[10]);
        return run([&] { return f(at_of(q), at_of(k), at_of(v), (const int32_t*)at_of(off), at_of(out), (float*)at_of(lse), &s, st); });
    });
}
// (function address, q, k, v, out, dout, lse, offsets, delta, dq, dk, dv, max_len, scale, device, stream)
ENTRY(packed_bwd) {
    return guarded(n, 16, [&] {
        const auto f = reinterpret_cast<decltype(&sa_attn_packed_bwd)>(address(a[0]));
        const Call on(a[14]);
        const at::Tensor &q = on(a[1]), &k = on(a[2]), &v = on(a[3]), &out = on(a[4]), &dout = on(a[5]), &lse = on(a[6]), &off = on.ids(a[7], OFFSETS),
                         &delta = on(a[8]), &dq = on(a[9]), &dk = on(a[10]), &dv = on(a[11]);
        const sa_packed s = packed_of(q, k, v, off, lse, a[12], a[13]);
        for (const at::Tensor* t : {&out, &dout, &dq}) same(*t, q, "out, dout and dq must have q's shape, type and strides");
        for (const at::Tensor* t : {&dk, &dv}) same(*t, k, "dk and dv must have k's shape, type and strides");
        same(delta, lse, "delta must have lse's shape, type and strides");
        void* st = stream(a[15]);
        return run([&] {
            return f(at_of(q), at_of(k), at_of(v), at_of(out), at_of(dout), (const float*)at_of(lse), (const int32_t*)at_of(off), (float*)at_of(delta),
                     at_of(dq), at_of(dk), at_of(dv), &s, st);
        });
    });
}
// (function address, q, k, v, offsets, out, lse, max_len, window, sinks, scale, device, stream)
ENTRY(window_fwd) {
    return guarded(n, 13, [&] {
        const auto f = reinterpret_cast<decltype(&sa_attn_window_fwd)>(address(a[0]));
        const Call on(a[11]);
        const at::Tensor &q = on(a[1]), &k = on(a[2]), &v = on(a[3]), &off = on.ids(a[4], OFFSETS), &out = on(a[5]), &lse = on(a[6]);
        const sa_packed s = packed_of(q, k, v, off, lse, a[7], a[10]);
        const sa_window w = {bound(a[8]), bound(a[9])};
        same(out, q, "out must have q's shape, type and strides");
        void* st = stream(a[12]);
        return run([&] { return f(at_of(q), at_of(k), at_of(v), (const int32_t*)at_of(off), at_of(out), (float*)at_of(lse), &s, &w, st); });
    });
}
// (function address, q, k, offsets, max_len, window, sinks): bytes
ENTRY(window_bwd_workspace) {
    return guarded(n, 7, [&] {
        const auto f = reinterpret_cast<decltype(&sa_attn_window_bwd_workspace)>(address(a[0]));
        const at::Tensor &q = tensor(a[1]), &k = tensor(a[2]), &off = tensor(a[3]);
        const Strides qs = strides(q), ks = strides(k);
        if (off.dim() != 1 || off.size(0) < 1) refuse(PyExc_ValueError, "offsets must hold one more number than there are sequences");
        const sa_packed s = {size(off, 0) - 1, size(q, 0), bound(a[4]), size(q, 1), size(k, 1), size(q, 2), qs.h, qs.s, ks.h, ks.s, q.size(0), type_of(q), 0.f};
        const sa_window w = {bound(a[5]), bound(a[6])};
        return PyLong_FromLongLong(f(&s, &w));
    });
}
// (function address, q, k, v, out, dout, lse, offsets, delta, dq, dk, dv, workspace, max_len, window, sinks, scale, device, stream)
ENTRY(window_bwd) {
    return guarded(n, 19, [&] {
        const auto f = reinterpret_cast<decltype(&sa_attn_window_bwd)>(address(a[0]));
        const Call on(a[17]);
        const at::Tensor &q = on(a[1]), &k = on(a[2]), &v = on(a[3]), &out = on(a[4]), &dout = on(a[5]), &lse = on(a[6]), &off = on.ids(a[7], OFFSETS),
                         &delta = on(a[8]), &dq = on(a[9]), &dk = on(a[10]), &dv = on(a[11]);
        const at::Tensor* work = maybe(on, a[12]);
        const sa_packed s = packed_of(q, k, v, off, lse, a[13], a[16]);
        const sa_window w = {bound(a[14]), bound(a[15])};
        for (const at::Tensor* t : {&out, &dout, &dq}) same(*t, q, "out, dout and dq must have q's shape, type and strides");
        for (const at::Tensor* t : {&dk, &dv}) same(*t, k, "dk and dv must have k's shape, type and strides");
        same(delta, lse, "delta must have lse's shape, type and strides");
        if (work && !work->is_contiguous()) refuse(PyExc_ValueError, "workspace must be contiguous");
        const int64_t bytes = work ? work->numel() * work->element_size() : 0;
        void* st = stream(a[18]);
        return run([&] {
            return f(at_of(q), at_of(k), at_of(v), at_of(out), at_of(dout), (const float*)at_of(lse), (const int32_t*)at_of(off), (float*)at_of(delta),
                     at_of(dq), at_of(dk), at_of(dv), at_of(work), bytes, &s, &w, st);
        });
    });
}
// [pages, page_size, heads, d]
sa_cache cache_of(const at::Tensor& k) {
    if (k.dim() != 4) refuse(PyExc_ValueError, "a cache is [pages, page size, heads, d]");
    if (k.size(3) > 1 && k.stride(3) != 1) refuse(PyExc_ValueError, "the head dimension must be contiguous");
    // (of a single head or page whatever fits)
    const int64_t h = k.size(2) == 1 ? k.size(3) : k.stride(2);
    return {size(k, 0), size(k, 1), size(k, 2), size(k, 3), k.size(0) == 1 ? 0 : k.stride(0), k.stride(1), h, type_of(k)};
}
// (function address, k, v, slot, k_cache, v_cache, pos, k_out, q, q_out, base, device, stream)
ENTRY(append) {
    return guarded(n, 13, [&] {
        const auto f = reinterpret_cast<decltype(&sa_cache_append)>(address(a[0]));
        const Call on(a[11]);
        const at::Tensor &k = on(a[1]), &v = on(a[2]), &slot = on.ids(a[3], "slot must be a contiguous int32 tensor"), &kc = on(a[4]), &vc = on(a[5]);
        const at::Tensor* pos = a[6] == Py_None ? nullptr : &on.ids(a[6], "pos must be a contiguous int32 tensor");
        const at::Tensor *k_out = maybe(on, a[7]), *q = maybe(on, a[8]), *q_out = maybe(on, a[9]);
        const Strides ks = strides(k);
        same(v, k, "k and v must have the same shape, type and strides");
        if (k_out) same(*k_out, k, "k_out must have k's shape, type and strides");
        same(vc, kc, "the caches must have the same shape, type and strides");
        const sa_cache cache = cache_of(kc);
        if (k.size(1) != cache.H_kv || k.size(2) != cache.d || k.scalar_type() != kc.scalar_type())
            refuse(PyExc_ValueError, "k and v must have the cache's heads, head dimension and type");
        const int64_t rows = k.size(0);
        if (slot.dim() != 1 || slot.size(0) != rows || (pos && (pos->dim() != 1 || pos->size(0) != rows)))
            refuse(PyExc_ValueError, "slot and pos must hold one number a row");
        sa_append r = {size(k, 0), 0, 0, 0, ks.h, ks.s, real(a[10])};
        if (q) {
            if (!q_out) refuse(PyExc_ValueError, "q is given without q_out");
            if (!pos) refuse(PyExc_ValueError, "q is given without pos");
            const Strides qs = strides(*q);
            if (q->size(0) != rows || q->size(2) != cache.d || q->scalar_type() != k.scalar_type())
                refuse(PyExc_ValueError, "q must have k's rows, head dimension and type");
            same(*q_out, *q, "q_out must have q's shape, type and strides");
            r.H = size(*q, 1);
            r.stride_h = qs.h;
            r.stride_s = qs.s;
        } else if (q_out) {
            refuse(PyExc_ValueError, "q_out is given without q");
        }
        void* st = stream(a[12]);
        return run([&] {
            return f(at_of(q), at_of(q_out), at_of(k), at_of(k_out), at_of(v), (const int32_t*)at_of(pos), (const int32_t*)at_of(slot), at_of(kc), at_of(vc),
                     &r, &cache, st);
        });
    });
}
sa_decode decode_of(const at::Tensor& q, const sa_cache& cache) {
    const Strides qs = strides(q);
    if (q.size(2) != cache.d || type_of(q) != cache.dtype) refuse(PyExc_ValueError, "q must have the cache's head dimension and type");
    return {size(q, 0), size(q, 1), 0, qs.s, qs.h, q.size(1), 0, 0.f};
}
// (function address, q, k_cache): bytes
ENTRY(decode_workspace) {
    return guarded(n, 3, [&] {
        const auto f = reinterpret_cast<decltype(&sa_attn_decode_workspace)>(address(a[0]));
        const sa_cache cache = cache_of(tensor(a[2]));
        const sa_decode s = decode_of(tensor(a[1]), cache);
        return PyLong_FromLongLong(f(&s, &cache));
    });
}
const char* const CACHES = "the caches must have the same shape, type and strides";
const char* const LENS = "lens must be a contiguous int32 tensor";
// page numbers of n sequences
void table_of(const at::Tensor& table, int64_t n, int32_t& max_pages, int64_t& stride) {
    if (table.scalar_type() != at::kInt || table.dim() != 2 || table.size(0) != n || (table.size(1) > 1 && table.stride(1) != 1))
        refuse(PyExc_ValueError, "table must be int32 [sequences, pages], pages contiguous");
    max_pages = size(table, 1);
    stride = n > 1 ? table.stride(0) : max_pages;
}
// one number for each of n
void numbers(const at::Tensor& t, int64_t n, const char* why) {
    if (t.dim() != 1 || t.size(0) != n) refuse(PyExc_ValueError, why);
}
int64_t bytes_of(const at::Tensor& work) {
    if (!work.is_contiguous()) refuse(PyExc_ValueError, "workspace must be contiguous");
    return work.numel() * work.element_size();
}
// (function address, q, k_cache, v_cache, table, lens, out, lse, workspace, scale, device, stream; with a window, window and sinks before scale)
template <bool WINDOW>
PyObject* decode_call(PyObject* const* a, Py_ssize_t n) {
    return guarded(n, WINDOW ? 14 : 12, [&] {
        PyObject* const* z = a + (WINDOW ? 11 : 9);         // scale, device, stream
        const Call on(z[1]);
        const at::Tensor &q = on(a[1]), &kc = on(a[2]), &vc = on(a[3]), &table = on(a[4]), &lens = on.ids(a[5], LENS), &out = on(a[6]), &work = on(a[8]);
        const at::Tensor* lse = maybe(on, a[7]);
        same(vc, kc, CACHES);
        same(out, q, "out must have q's shape, type and strides");
        const sa_cache cache = cache_of(kc);
        sa_decode s = decode_of(q, cache);
        table_of(table, q.size(0), s.max_pages, s.table_stride);
        numbers(lens, q.size(0), "lens must hold one number a sequence");
        if (lse) {
            statistics(*lse, q.size(0), q.size(1), "lse must be float32 [sequences, heads], heads contiguous");
            if (q.size(0) > 1) s.stat_stride_b = lse->stride(0);
        }
        const int64_t bytes = bytes_of(work);
        s.softmax_scale = real(z[0]);
        sa_window w = {0, 0};
        if (WINDOW) w = {bound(a[9]), bound(a[10])};
        void* st = stream(z[2]);
        return run([&] {
            if constexpr (WINDOW)
                return reinterpret_cast<decltype(&sa_attn_window_decode)>(address(a[0]))(
                    at_of(q), at_of(kc), at_of(vc), (const int32_t*)at_of(table), (const int32_t*)at_of(lens), at_of(out), (float*)at_of(lse), at_of(work),
                    bytes, &s, &cache, &w, st);
            else
                return reinterpret_cast<decltype(&sa_attn_decode)>(address(a[0]))(
                    at_of(q), at_of(kc), at_of(vc), (const int32_t*)at_of(table), (const int32_t*)at_of(lens), at_of(out), (float*)at_of(lse), at_of(work),
                    bytes, &s, &cache, st);
        });
    });
}
ENTRY(decode) { return decode_call<false>(a, n); }
ENTRY(window_decode) { return decode_call<true>(a, n); }
// q [sequences, drafted tokens, heads, d]
sa_tree tree_of(const at::Tensor& q, const sa_cache& cache) {
    if (q.dim() != 4) refuse(PyExc_ValueError, "expected [sequences, drafted tokens, heads, d]");
    if (q.size(3) > 1 && q.stride(3) != 1) refuse(PyExc_ValueError, "the head dimension must be contiguous");
    if (q.size(3) != cache.d || type_of(q) != cache.dtype) refuse(PyExc_ValueError, "q must have the cache's head dimension and type");
    // (of a single sequence, token or head whatever fits)
    const int64_t h = q.size(2) == 1 ? q.size(3) : q.stride(2), t = q.size(1) <= 1 ? h * q.size(2) : q.stride(1), b = q.size(0) <= 1 ? t * q.size(1) : q.stride(0);
    return {size(q, 0), size(q, 1), size(q, 2), 0, b, t, h, q.size(1) * q.size(2), q.size(2), 0, q.size(1), 0.f};
}
// (function address, q, k_cache): bytes
ENTRY(tree_workspace) {
    return guarded(n, 3, [&] {
        const auto f = reinterpret_cast<decltype(&sa_attn_tree_workspace)>(address(a[0]));
        const sa_cache cache = cache_of(tensor(a[2]));
        const sa_tree s = tree_of(tensor(a[1]), cache);
        return PyLong_FromLongLong(f(&s, &cache));
    });
}
// (function address, q, k_cache, v_cache, table, lens, drafts, seen, out, lse, workspace, scale, device, stream)
ENTRY(tree) {
    return guarded(n, 14, [&] {
        const auto f = reinterpret_cast<decltype(&sa_attn_tree)>(address(a[0]));
        const Call on(a[12]);
        const at::Tensor &q = on(a[1]), &kc = on(a[2]), &vc = on(a[3]), &table = on(a[4]), &lens = on.ids(a[5], LENS), &seen = on(a[7]), &out = on(a[8]),
                         &work = on(a[10]);
        const at::Tensor* drafts = a[6] == Py_None ? nullptr : &on.ids(a[6], "drafts must be a contiguous int32 tensor");
        const at::Tensor* lse = maybe(on, a[9]);
        same(vc, kc, CACHES);
        same(out, q, "out must have q's shape, type and strides");
        const sa_cache cache = cache_of(kc);
        sa_tree s = tree_of(q, cache);
        const int64_t B = q.size(0), T = q.size(1), H = q.size(2);
        table_of(table, B, s.max_pages, s.table_stride);
        numbers(lens, B, "lens must hold one number a sequence");
        if (drafts) numbers(*drafts, B, "drafts must hold one number a sequence");
        if (seen.scalar_type() != at::kLong || seen.dim() != 2 || seen.size(0) != B || seen.size(1) != T || (T > 1 && seen.stride(1) != 1))
            refuse(PyExc_ValueError, "seen must be int64 [sequences, drafted tokens], tokens contiguous");
        if (B > 1) s.seen_stride = seen.stride(0);
        if (lse) {
            if (lse->scalar_type() != at::kFloat || lse->dim() != 3 || lse->size(0) != B || lse->size(1) != T || lse->size(2) != H || (H > 1 && lse->stride(2) != 1))
                refuse(PyExc_ValueError, "lse must be float32 [sequences, drafted tokens, heads], heads contiguous");
            if (T > 1) s.stat_stride_t = lse->stride(1);
            s.stat_stride_b = B > 1 ? lse->stride(0) : T * s.stat_stride_t;
        }
        const int64_t bytes = bytes_of(work);
        s.softmax_scale = real(a[11]);
        void* st = stream(a[13]);
        return run([&] {
            return f(at_of(q), at_of(kc), at_of(vc), (const int32_t*)at_of(table), (const int32_t*)at_of(lens), (const int32_t*)at_of(drafts),
                     (const int64_t*)at_of(seen), at_of(out), (float*)at_of(lse), at_of(work), bytes, &s, &cache, st);
        });
    });
}
// (function address, k_cache, v_cache, table, lens, chosen, accepted, lens_after, device, stream)
ENTRY(accept) {
    return guarded(n, 10, [&] {
        const auto f = reinterpret_cast<decltype(&sa_cache_accept)>(address(a[0]));
        const Call on(a[8]);
        const at::Tensor &kc = on(a[1]), &vc = on(a[2]), &table = on(a[3]), &lens = on.ids(a[4], LENS), &chosen = on(a[5]),
                         &accepted = on.ids(a[6], "accepted must be a contiguous int32 tensor");
        const at::Tensor* after = a[7] == Py_None ? nullptr : &on.ids(a[7], "lens_after must be a contiguous int32 tensor");
        same(vc, kc, CACHES);
        const sa_cache cache = cache_of(kc);
        const int64_t B = lens.dim() == 1 ? lens.size(0) : -1;
        numbers(lens, B, "lens must hold one number a sequence");
        numbers(accepted, B, "accepted must hold one number a sequence");
        if (after) numbers(*after, B, "lens_after must hold one number a sequence");
        if (chosen.scalar_type() != at::kInt || chosen.dim() != 2 || chosen.size(0) != B || (chosen.size(1) > 1 && chosen.stride(1) != 1))
            refuse(PyExc_ValueError, "chosen must be int32 [sequences, drafted tokens], tokens contiguous");
        sa_accept s = {size(lens, 0), size(chosen, 1), 0, 0, B > 1 ? chosen.stride(0) : chosen.size(1)};
        table_of(table, B, s.max_pages, s.table_stride);
        void* st = stream(a[9]);
        return run([&] {
            return f(at_of(kc), at_of(vc), (const int32_t*)at_of(table), (const int32_t*)at_of(lens), (const int32_t*)at_of(chosen),
                     (const int32_t*)at_of(accepted), (int32_t*)at_of(after), &s, &cache, st);
        });
    });
}
// (function address, k_cache, v_cache, from, to, tokens, device, stream)
ENTRY(copy) {
    return guarded(n, 8, [&] {
        const auto f = reinterpret_cast<decltype(&sa_cache_copy)>(address(a[0]));
        const Call on(a[6]);
        const at::Tensor &kc = on(a[1]), &vc = on(a[2]), &from = on.ids(a[3], "src must be a contiguous int32 tensor"),
                         &to = on.ids(a[4], "dst must be a contiguous int32 tensor");
        const at::Tensor* tokens = a[5] == Py_None ? nullptr : &on.ids(a[5], "tokens must be a contiguous int32 tensor");
        same(vc, kc, CACHES);
        const sa_cache cache = cache_of(kc);
        numbers(to, from.dim() == 1 ? from.size(0) : -1, "src and dst must hold as many page numbers");
        if (tokens) numbers(*tokens, from.size(0), "tokens must hold one number a page");
        const int32_t pages = size(from, 0);
        void* st = stream(a[7]);
        return run([&] {
            return f(at_of(kc), at_of(vc), (const int32_t*)at_of(from), (const int32_t*)at_of(to), (const int32_t*)at_of(tokens), pages, &cache, st);
        });
    });
}
// (the type of a shape, a function that makes an integer of what is none)
ENTRY(set_up) {
    return guarded(n, 2, [&]() -> PyObject* {
        if (!PyType_Check(a[0]) || !PyCallable_Check(a[1])) {
            PyErr_SetString(PyExc_TypeError, "expected a type and a function");
            return nullptr;
        }
        Py_INCREF(a[0]);
        Py_INCREF(a[1]);
        shape_type = reinterpret_cast<PyTypeObject*>(a[0]);
        other_integer = a[1];
        Py_RETURN_NONE;
    });
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(two), FAST(three), FAST(step_fwd), FAST(step_bwd), FAST(ring_fwd), FAST(ring_bwd), FAST(rope),
                         FAST(permute), FAST(packed_fwd), FAST(packed_bwd), FAST(window_fwd), FAST(window_bwd), FAST(window_bwd_workspace), FAST(append), FAST(decode), FAST(decode_workspace), FAST(window_decode), FAST(tree), FAST(tree_workspace), FAST(accept), FAST(copy),
                         FAST(extent_of), FAST(set_up), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }

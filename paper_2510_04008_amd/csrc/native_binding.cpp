// CPython extension `_native`: argument marshalling of the entry points a training or serving loop calls for every layer
// and token.  Small calls are bound by the host: checking ten tensors and building fifteen ctypes arguments in Python costs
// 10-20 us, more than the kernels of a short pass take; here it is 1-2 us.  No arithmetic of the layer and no torch types
// beyond this file: the library behind it is the plain C ABI.
//
// Every function takes positional arguments only, raises ValueError for a tensor that is not what the descriptor says, and
// returns the library's status code.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <string>
#include <vector>

#include "race_attn.h"

namespace {

struct BadArgument {};                      // a Python exception has been set

struct Desc {
    race_attn_desc_t d;
    explicit Desc(PyObject *o)
    {
        Py_buffer view;
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw BadArgument{};
        const bool ok = view.len == static_cast<Py_ssize_t>(sizeof d);
        if (ok) std::memcpy(&d, view.buf, sizeof d);
        PyBuffer_Release(&view);
        if (!ok) {
            PyErr_SetString(PyExc_TypeError, "desc must be a RaceAttnDesc");
            throw BadArgument{};
        }
    }
    at::ScalarType elem() const { return d.dtype == RACE_F32 ? at::kFloat : at::kBFloat16; }
    int32_t heads() const { return d.N == 0 ? 0 : d.H; }       // seeds that a pass over the sequence reads
};

struct Shape { int n; int64_t s[5]; };

void *tensor(PyObject *o, const char *name, const Shape &shape, at::ScalarType type)
{
    if (THPVariable_Check(o)) {
        const at::Tensor &t = THPVariable_Unpack(o);
        bool ok = t.is_cuda() && t.scalar_type() == type && t.dim() == shape.n && t.is_contiguous();
        for (int i = 0; ok && i < shape.n; ++i) ok = t.size(i) == shape.s[i];
        if (ok) return t.data_ptr();
    }
    std::string want;
    for (int i = 0; i < shape.n; ++i) want += (i ? ", " : "") + std::to_string(shape.s[i]);
    PyErr_Format(PyExc_ValueError, "%s must be a contiguous device tensor of shape (%s) and dtype %s", name, want.c_str(),
                 type == at::kFloat ? "torch.float32" : type == at::kLong ? "torch.int64" : "torch.bfloat16");
    throw BadArgument{};
}
Shape full(const Desc &d) { return Shape{4, {d.d.B, d.d.H, d.d.N, d.d.d}}; }
Shape rows(const Desc &d) { return Shape{3, {d.d.B, d.d.H, d.d.d}}; }
Shape per_token(const Desc &d) { return Shape{3, {d.d.B, d.d.H, d.d.N}}; }
Shape per_head(const Desc &d) { return Shape{2, {d.d.B, d.d.H}}; }
Shape state_shape(const Desc &d)
{
    return Shape{5, {d.d.B, d.d.H, d.d.L, (d.d.P >= 0 && d.d.P < 31) ? int64_t(1) << d.d.P : 0, int64_t(d.d.d) + 1}};
}

struct Workspace {
    void *ptr = nullptr;
    size_t bytes = 0;
    explicit Workspace(PyObject *o)
    {
        if (o == Py_None) return;
        if (!THPVariable_Check(o)) {
            PyErr_SetString(PyExc_ValueError, "workspace must be a device tensor");
            throw BadArgument{};
        }
        const at::Tensor &t = THPVariable_Unpack(o);
        ptr = t.data_ptr();
        bytes = static_cast<size_t>(t.numel()) * t.element_size();
    }
};

// int(s) modulo 2^64 of every element (any number, not integers only).  needed: how many the call reads (an empty sequence
// needs none); None is for the decoding step alone.
struct Seeds {
    std::vector<uint64_t> v;
    const uint64_t *ptr = nullptr;
    Seeds(PyObject *o, int32_t needed, bool optional = false)
    {
        if (optional && o == Py_None) return;
        PyObject *fast = PySequence_Fast(o, "proj_seeds must be a sequence of integers");
        if (!fast) throw BadArgument{};
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast);
        v.resize(n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            PyObject *num = PyNumber_Long(PySequence_Fast_GET_ITEM(fast, i));
            if (num) {
                v[i] = PyLong_AsUnsignedLongLongMask(num);
                Py_DECREF(num);
            }
            if (PyErr_Occurred()) {
                Py_DECREF(fast);
                throw BadArgument{};
            }
        }
        Py_DECREF(fast);
        if (n < needed) {
            PyErr_Format(PyExc_ValueError, "proj_seeds must have one seed per head (%d)", static_cast<int>(needed));
            throw BadArgument{};
        }
        ptr = v.data();
    }
};

race_stream_t stream_of(PyObject *o)
{
    if (o == Py_None) return reinterpret_cast<race_stream_t>(c10::hip::getCurrentHIPStream().stream());
    PyObject *raw = PyObject_HasAttrString(o, "cuda_stream") ? PyObject_GetAttrString(o, "cuda_stream") : (Py_INCREF(o), o);
    if (!raw) throw BadArgument{};
    PyObject *num = PyNumber_Long(raw);
    Py_DECREF(raw);
    if (!num) throw BadArgument{};
    void *p = PyLong_AsVoidPtr(num);
    Py_DECREF(num);
    if (PyErr_Occurred()) throw BadArgument{};
    return reinterpret_cast<race_stream_t>(p);
}

// Other Python threads run while the library works (the first call with new seeds expands W; a full queue makes a launch wait).
struct ReleaseGil {
    PyThreadState *saved = PyEval_SaveThread();
    ~ReleaseGil() { PyEval_RestoreThread(saved); }
};

template <int N, typename F>
PyObject *call(PyObject *const *args, Py_ssize_t nargs, F f)
{
    if (nargs != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", N, nargs);
        return nullptr;
    }
    try {
        return PyLong_FromLong(f(args));
    } catch (const BadArgument &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// (desc, Q, K, V, seeds, O, den, workspace, stream); workspace None: the library's built-in scratch
PyObject *fwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return call<9>(args, n, [](PyObject *const *a) {
        const Desc d(a[0]);
        const Shape t = full(d);
        const at::ScalarType e = d.elem();
        void *Q = tensor(a[1], "Q", t, e), *K = tensor(a[2], "K", t, e), *V = tensor(a[3], "V", t, e);
        const Seeds s(a[4], d.heads());
        void *O = tensor(a[5], "O", t, e);
        float *den = static_cast<float *>(tensor(a[6], "den", per_token(d), at::kFloat));
        const race_stream_t st = stream_of(a[8]);
        const bool built_in = a[7] == Py_None;
        const Workspace ws(a[7]);
        const ReleaseGil released;
        if (built_in) return race_attn_fwd_static(&d.d, Q, K, V, s.ptr, O, den, st);
        return race_attn_fwd(&d.d, Q, K, V, s.ptr, O, den, ws.ptr, ws.bytes, st);
    });
}

// (desc, Q, K, V, O, den, dO, seeds, dQ, dK, dV, dbeta or None, workspace, stream, saved)
PyObject *bwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return call<15>(args, n, [](PyObject *const *a) {
        const Desc d(a[0]);
        const Shape t = full(d);
        const at::ScalarType e = d.elem();
        void *Q = tensor(a[1], "Q", t, e), *K = tensor(a[2], "K", t, e), *V = tensor(a[3], "V", t, e), *O = tensor(a[4], "O", t, e);
        const float *den = static_cast<float *>(tensor(a[5], "den", per_token(d), at::kFloat));
        void *dO = tensor(a[6], "dO", t, e);
        const Seeds s(a[7], d.heads());
        void *dQ = tensor(a[8], "dQ", t, e), *dK = tensor(a[9], "dK", t, e), *dV = tensor(a[10], "dV", t, e);
        float *dbeta = a[11] == Py_None ? nullptr : static_cast<float *>(tensor(a[11], "dbeta", per_head(d), at::kFloat));
        const Workspace ws(a[12]);
        const race_stream_t st = stream_of(a[13]);
        const auto entry = a[14] == Py_True ? race_attn_bwd_saved : race_attn_bwd_beta;
        const ReleaseGil released;
        return entry(&d.d, Q, K, V, O, den, dO, s.ptr, dQ, dK, dV, dbeta, ws.ptr, ws.bytes, st);
    });
}

// (desc, K or None, V or None, seeds, state, workspace or None, stream)
PyObject *state_init(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return call<7>(args, n, [](PyObject *const *a) {
        const Desc d(a[0]);
        float *state = static_cast<float *>(tensor(a[4], "state", state_shape(d), at::kFloat));
        void *K = nullptr, *V = nullptr;
        if (d.d.N > 0) {
            K = tensor(a[1], "K", full(d), d.elem());
            V = tensor(a[2], "V", full(d), d.elem());
        }
        const Seeds s(a[3], d.heads());
        const Workspace ws(a[5]);
        const race_stream_t st = stream_of(a[6]);
        const ReleaseGil released;
        return race_attn_state_init(&d.d, K, V, s.ptr, state, ws.ptr, ws.bytes, st);
    });
}

// (desc, q, k, v, seeds or None, state, o, den, workspace, stream)
PyObject *step(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return call<10>(args, n, [](PyObject *const *a) {
        const Desc d(a[0]);
        const Shape r = rows(d);
        const at::ScalarType e = d.elem();
        void *q = tensor(a[1], "q", r, e), *k = tensor(a[2], "k", r, e), *v = tensor(a[3], "v", r, e);
        const Seeds s(a[4], d.d.H, true);
        float *state = static_cast<float *>(tensor(a[5], "state", state_shape(d), at::kFloat));
        void *o = tensor(a[6], "o", r, e);
        float *den = static_cast<float *>(tensor(a[7], "den", per_head(d), at::kFloat));
        const Workspace ws(a[8]);
        const race_stream_t st = stream_of(a[9]);
        const ReleaseGil released;
        return race_attn_step(&d.d, q, k, v, s.ptr, state, o, den, ws.ptr, ws.bytes, st);
    });
}

// ---------------------------------------------------------------- the gated delta rule, rows of queries and keys
template <class D>
D plain_desc(PyObject *o, const char *type)
{
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw BadArgument{};
    D d;
    const bool ok = view.len == static_cast<Py_ssize_t>(sizeof d);
    if (ok) std::memcpy(&d, view.buf, sizeof d);
    PyBuffer_Release(&view);
    if (!ok) {
        PyErr_Format(PyExc_TypeError, "desc must be a %s", type);
        throw BadArgument{};
    }
    return d;
}
at::ScalarType elem_of(int32_t dtype) { return dtype == RACE_F32 ? at::kFloat : at::kBFloat16; }

// Tensors of one call: contiguous, of the current device (its stream is the one that they are used on).
struct Call {
    const int device = c10::hip::current_device();
    void on_device(const at::Tensor &t, const char *name) const
    {
        if (t.get_device() == device) return;
        PyErr_Format(PyExc_ValueError, "%s is on device %d, the current device is %d", name, static_cast<int>(t.get_device()), device);
        throw BadArgument{};
    }
    void *operator()(PyObject *o, const char *name, const Shape &shape, at::ScalarType type) const
    {
        void *p = tensor(o, name, shape, type);
        on_device(THPVariable_Unpack(o), name);
        return p;
    }
    float *floats(PyObject *o, const char *name, const Shape &shape) const { return static_cast<float *>((*this)(o, name, shape, at::kFloat)); }
    float *maybe(PyObject *o, const char *name, const Shape &shape) const { return o == Py_None ? nullptr : floats(o, name, shape); }
    Workspace workspace(PyObject *o) const
    {
        const Workspace w(o);
        if (o == Py_None) return w;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda() || !t.is_contiguous()) {
            PyErr_SetString(PyExc_ValueError, "workspace must be a contiguous device tensor");
            throw BadArgument{};
        }
        on_device(t, "workspace");
        return w;
    }
    // rows (B, N, heads, d), the elements of a row together; their strides
    void *rows(PyObject *o, const char *name, const Shape &shape, at::ScalarType type, int64_t *strides) const
    {
        if (THPVariable_Check(o)) {
            const at::Tensor &t = THPVariable_Unpack(o);
            bool ok = t.is_cuda() && t.scalar_type() == type && t.dim() == 4 && t.stride(3) == 1;
            for (int i = 0; ok && i < 4; ++i) ok = t.size(i) == shape.s[i];
            if (ok) {
                on_device(t, name);
                for (int i = 0; i < 3; ++i) strides[i] = t.stride(i);
                return t.data_ptr();
            }
        }
        PyErr_Format(PyExc_ValueError, "%s must be a device tensor of shape (%lld, %lld, %lld, %lld) and dtype %s with stride 1 in its last dimension", name,
                     static_cast<long long>(shape.s[0]), static_cast<long long>(shape.s[1]), static_cast<long long>(shape.s[2]),
                     static_cast<long long>(shape.s[3]), type == at::kFloat ? "torch.float32" : "torch.bfloat16");
        throw BadArgument{};
    }
};

struct DeltaShapes {
    Shape qk, v, gates, state;
    DeltaShapes(const race_delta_desc_t &d, bool step)
    {
        const int64_t B = d.B, H = d.H, Hk = d.Hk, N = d.N, dk = d.dk, dv = d.dv;
        qk = step ? Shape{3, {B, Hk, dk}} : Shape{4, {B, Hk, N, dk}};
        v = step ? Shape{3, {B, H, dv}} : Shape{4, {B, H, N, dv}};
        gates = step ? Shape{2, {B, H}} : Shape{3, {B, H, N}};
        state = Shape{4, {B, H, dk, dv}};
    }
};

// (desc, Q, K, V, g, beta, state_in or None, O, state_out or None, workspace, stream)
PyObject *delta_fwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return call<11>(args, n, [](PyObject *const *a) {
        const auto d = plain_desc<race_delta_desc_t>(a[0], "RaceDeltaDesc");
        const DeltaShapes s(d, false);
        const at::ScalarType e = elem_of(d.dtype);
        const Call t;
        void *Q = t(a[1], "Q", s.qk, e), *K = t(a[2], "K", s.qk, e), *V = t(a[3], "V", s.v, e);
        const float *g = t.floats(a[4], "g", s.gates), *beta = t.floats(a[5], "beta", s.gates), *in = t.maybe(a[6], "state_in", s.state);
        void *O = t(a[7], "O", s.v, e);
        float *out = t.maybe(a[8], "state_out", s.state);
        const Workspace ws = t.workspace(a[9]);
        const race_stream_t st = stream_of(a[10]);
        const ReleaseGil released;
        return race_delta_fwd(&d, Q, K, V, g, beta, in, O, out, ws.ptr, ws.bytes, st);
    });
}

// (desc, Q, K, V, g, beta, state_in or None, dO, dstate_out or None, dQ, dK, dV, dg, dbeta, dstate_in or None, workspace, stream)
PyObject *delta_bwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return call<17>(args, n, [](PyObject *const *a) {
        const auto d = plain_desc<race_delta_desc_t>(a[0], "RaceDeltaDesc");
        const DeltaShapes s(d, false);
        const at::ScalarType e = elem_of(d.dtype);
        const Call t;
        void *Q = t(a[1], "Q", s.qk, e), *K = t(a[2], "K", s.qk, e), *V = t(a[3], "V", s.v, e);
        const float *g = t.floats(a[4], "g", s.gates), *beta = t.floats(a[5], "beta", s.gates), *in = t.maybe(a[6], "state_in", s.state);
        void *dO = t(a[7], "dO", s.v, e);
        const float *dout = t.maybe(a[8], "dstate_out", s.state);
        void *dQ = t(a[9], "dQ", s.qk, e), *dK = t(a[10], "dK", s.qk, e), *dV = t(a[11], "dV", s.v, e);
        float *dg = t.floats(a[12], "dg", s.gates), *dbeta = t.floats(a[13], "dbeta", s.gates), *din = t.maybe(a[14], "dstate_in", s.state);
        const Workspace ws = t.workspace(a[15]);
        const race_stream_t st = stream_of(a[16]);
        const ReleaseGil released;
        return race_delta_bwd(&d, Q, K, V, g, beta, in, dO, dout, dQ, dK, dV, dg, dbeta, din, ws.ptr, ws.bytes, st);
    });
}

// (desc, q, k, v, g, beta, state, o, stream)
PyObject *delta_step(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return call<9>(args, n, [](PyObject *const *a) {
        const auto d = plain_desc<race_delta_desc_t>(a[0], "RaceDeltaDesc");
        const DeltaShapes s(d, true);
        const at::ScalarType e = elem_of(d.dtype);
        const Call t;
        void *q = t(a[1], "q", s.qk, e), *k = t(a[2], "k", s.qk, e), *v = t(a[3], "v", s.v, e);
        const float *g = t.floats(a[4], "g", s.gates), *beta = t.floats(a[5], "beta", s.gates);
        float *state = t.floats(a[6], "state", s.state);
        void *o = t(a[7], "o", s.v, e);
        const race_stream_t st = stream_of(a[8]);
        const ReleaseGil released;
        return race_delta_step(&d, q, k, v, g, beta, state, o, st);
    });
}

struct Rotary {
    race_rotary_desc_t d;
    const Call t;
    at::ScalarType e;
    const void *q, *k = nullptr;
    const float *wq, *wk = nullptr;
    double freq[128];
    const int64_t *positions = nullptr;
    // desc, q, k or None, wq or None, wk or None, inv_freq, positions or None
    explicit Rotary(PyObject *const *a) : d(plain_desc<race_rotary_desc_t>(a[0], "RaceRotaryDesc")), e(elem_of(d.dtype))
    {
        q = t.rows(a[1], "q", given(d.Hq), e, d.q_strides);
        wq = t.maybe(a[3], "wq", Shape{1, {d.d}});
        if (d.Hk > 0) {
            k = t.rows(a[2], "k", given(d.Hk), e, d.k_strides);
            wk = t.maybe(a[4], "wk", Shape{1, {d.d}});
        }
        const Py_ssize_t need = d.rot / 2;
        PyObject *fast = need > 0 ? PySequence_Fast(a[5], "inv_freq must be a sequence of numbers") : nullptr;
        if (need > 0 && !fast) throw BadArgument{};
        if (need > 128 || (need > 0 && PySequence_Fast_GET_SIZE(fast) != need)) {
            Py_XDECREF(fast);
            PyErr_Format(PyExc_ValueError, "inv_freq must have rot / 2 (%d) elements", static_cast<int>(need));
            throw BadArgument{};
        }
        for (Py_ssize_t i = 0; i < need; ++i) freq[i] = PyFloat_AsDouble(PySequence_Fast_GET_ITEM(fast, i));
        Py_XDECREF(fast);
        if (PyErr_Occurred()) throw BadArgument{};
        if (a[6] != Py_None) positions = static_cast<const int64_t *>(t(a[6], "positions", Shape{2, {d.B, d.N}}, at::kLong));
    }
    Shape given(int64_t heads) const { return Shape{4, {d.B, d.N, heads, d.d}}; }
    Shape made(int64_t heads) const { return Shape{4, {d.B, heads, d.N, d.d}}; }
};

// (desc, q, k, wq, wk, inv_freq, positions, Q, K or None, stream)
PyObject *rotary_fwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return call<10>(args, n, [](PyObject *const *a) {
        const Rotary r(a);
        void *Q = r.t(a[7], "Q", r.made(r.d.Hq), r.e), *K = r.d.Hk > 0 ? r.t(a[8], "K", r.made(r.d.Hk), r.e) : nullptr;
        const race_stream_t st = stream_of(a[9]);
        const ReleaseGil released;
        return race_qk_rotary_fwd(&r.d, r.q, r.k, r.wq, r.wk, r.freq, r.positions, Q, K, st);
    });
}

// (desc, q, k, wq, wk, inv_freq, positions, dQ, dK or None, dq, dk or None, dwq or None, dwk or None, workspace or None, stream)
PyObject *rotary_bwd(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return call<15>(args, n, [](PyObject *const *a) {
        Rotary r(a);
        const bool keys = r.d.Hk > 0;
        void *dQ = r.t(a[7], "dQ", r.made(r.d.Hq), r.e), *dK = keys ? r.t(a[8], "dK", r.made(r.d.Hk), r.e) : nullptr;
        void *dq = r.t.rows(a[9], "dq", r.given(r.d.Hq), r.e, r.d.dq_strides), *dk = keys ? r.t.rows(a[10], "dk", r.given(r.d.Hk), r.e, r.d.dk_strides) : nullptr;
        float *dwq = r.t.maybe(a[11], "dwq", Shape{1, {r.d.d}}), *dwk = r.t.maybe(a[12], "dwk", Shape{1, {r.d.d}});
        const Workspace ws = r.t.workspace(a[13]);
        const race_stream_t st = stream_of(a[14]);
        const ReleaseGil released;
        return race_qk_rotary_bwd(&r.d, r.q, r.k, r.wq, r.wk, r.freq, r.positions, dQ, dK, dq, dk, dwq, dwk, ws.ptr, ws.bytes, st);
    });
}

#define ENTRY(name, doc) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(name)), METH_FASTCALL, doc}
PyMethodDef kMethods[] = {
    ENTRY(fwd, "race_attn_fwd, or race_attn_fwd_static without a workspace"),
    ENTRY(bwd, "race_attn_bwd_beta or race_attn_bwd_saved"),
    ENTRY(state_init, "race_attn_state_init"),
    ENTRY(step, "race_attn_step"),
    ENTRY(delta_fwd, "race_delta_fwd"),
    ENTRY(delta_bwd, "race_delta_bwd"),
    ENTRY(delta_step, "race_delta_step"),
    ENTRY(rotary_fwd, "race_qk_rotary_fwd"),
    ENTRY(rotary_bwd, "race_qk_rotary_bwd"),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_native", "argument marshalling of the RACE Attention entry points", -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&kModule); }

// fastcall.cpp -- the Python binding's argument marshalling in native code.
//
// A call through ctypes spends 12 - 16 us on the host (attribute reads, checks,
// two stream objects, sixteen argument conversions), more than most of the
// library's kernels run.  These functions read the same arguments, make the
// same checks and call the same C entry points in 2 - 3 us.  They handle the
// ordinary call only: on anything else -- a failed check, a tensor subclass,
// lengths that are not a list or tuple of ints, a workspace still to be
// allocated -- they return None without having enqueued anything, and the
// caller takes its Python path, which does the work or raises the error.  An
// int result is the C entry point's return code.  Nothing is kept between
// calls but the C functions' addresses.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstring>
#include <initializer_list>

#include "mad.h"

namespace {

struct Entry {
    decltype(&mad_draft_decode_attn) decode;
    decltype(&mad_draft_step_attn) step;
    decltype(&mad_memory_update) update;
    decltype(&mad_verify_attn) verify;
    decltype(&mad_verify_attn_vt) verify_vt;
    decltype(&mad_accept_greedy) greedy;
    decltype(&mad_accept_stochastic) stoch;
    decltype(&mad_rmsnorm_qkv_rope) qkv;
    decltype(&mad_linear_residual) linear;
    decltype(&mad_rmsnorm_swiglu) swiglu;
    decltype(&mad_workspace_bytes) ws_bytes;
    decltype(&mad_kv8_append) kv8_append;
    decltype(&mad_verify_attn_kv8) verify8;
    decltype(&mad_sample) sample;
    decltype(&mad_qk_norm_rope) norm_rope;
    decltype(&mad_kv4_append) kv4_append;
    decltype(&mad_verify_attn_kv4) verify4;
    decltype(&mad_token_logprobs) logprobs;
} g;
PyObject *g_kv, *g_kv8, *g_kv4, *g_ws, *g_stream;   // classes KV, KV8 and KV4, the default workspaces' dict, the raw-stream getter
PyObject *s_k, *s_v, *s_length, *s_start, *s_buf, *s_k_scale, *s_v_scale, *s_block;

struct Unhandled {};   // thrown for every call the Python path has to take
void need(bool ok) {
    if (!ok) throw Unhandled();
}

// an owned reference
struct Ref {
    PyObject *p;
    explicit Ref(PyObject *o) : p(o) { need(o != nullptr); }
    ~Ref() { Py_DECREF(p); }
    Ref(const Ref &) = delete;
};

const at::Tensor &tensor(PyObject *o) {
    need(THPVariable_CheckExact(o));
    return THPVariable_Unpack(o);
}
// a contiguous tensor on the call's device
const at::Tensor &dense(PyObject *o, const at::Device &dev) {
    const at::Tensor &t = tensor(o);
    need(t.is_contiguous() && t.device() == dev);
    return t;
}
const at::Tensor &first(PyObject *o) {
    const at::Tensor &t = tensor(o);
    need(t.is_contiguous() && t.is_cuda() && t.layout() == at::kStrided);
    return t;
}
bool shape(const at::Tensor &t, std::initializer_list<int64_t> want) { return t.sizes() == at::IntArrayRef(want); }
int dtype_code(const at::Tensor &t) {
    if (t.scalar_type() == at::kBFloat16) return MAD_BF16;
    need(t.scalar_type() == at::kFloat);
    return MAD_F32;
}
int small(int64_t v) {
    need(v >= 0 && v <= 0x7fffffff);
    return (int)v;
}
int as_int(PyObject *o) {
    need(PyLong_CheckExact(o));
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);
    need(!over && v >= INT32_MIN && v <= INT32_MAX);
    return (int)v;
}
double as_double(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    need(v != -1.0 || !PyErr_Occurred());
    return v;
}
// the n ints of a list or tuple
template <typename I> void ints(PyObject *o, int64_t n, I *out) {
    need((PyList_CheckExact(o) || PyTuple_CheckExact(o)) && PySequence_Fast_GET_SIZE(o) == n);
    PyObject **items = PySequence_Fast_ITEMS(o);
    for (int64_t i = 0; i < n; ++i) {
        const int v = as_int(items[i]);
        need(sizeof(I) == 4 || (v >= 0 && v <= 255));
        out[i] = (I)v;
    }
}

// What the types of the arguments alone say, looked at before anything is read: a call that is not an ordinary one
// for them goes back at once (0.2 us; an exception on the way costs 3, a fifth of the call on the Python path).
bool plain_ints(PyObject *o) {
    const Py_ssize_t n = PyList_CheckExact(o) || PyTuple_CheckExact(o) ? PySequence_Fast_GET_SIZE(o) : 0;
    return n > 0 && PyLong_CheckExact(PySequence_Fast_GET_ITEM(o, 0)) && PyLong_CheckExact(PySequence_Fast_GET_ITEM(o, n - 1));
}
bool plain_rows(PyObject *o) {   // [B][n] ints
    const Py_ssize_t n = PyList_CheckExact(o) || PyTuple_CheckExact(o) ? PySequence_Fast_GET_SIZE(o) : 0;
    return n > 0 && plain_ints(PySequence_Fast_GET_ITEM(o, 0));
}
bool plain_flags(PyObject *o) {   // ints or bools, or None
    if (o == Py_None) return true;
    const Py_ssize_t n = PyList_CheckExact(o) || PyTuple_CheckExact(o) ? PySequence_Fast_GET_SIZE(o) : 0;
    return n > 0 && (PyBool_Check(PySequence_Fast_GET_ITEM(o, 0)) || PyLong_CheckExact(PySequence_Fast_GET_ITEM(o, 0)));
}
bool plain_real(PyObject *o) { return PyFloat_CheckExact(o) || PyLong_CheckExact(o); }
bool plain_attr(PyObject *o, PyObject *name, bool none) {
    PyObject *v = PyObject_GetAttr(o, name);
    const bool ok = v && (v == Py_None ? none : plain_ints(v));
    Py_XDECREF(v);
    PyErr_Clear();
    return ok;
}
bool plain_kv(PyObject *o) {
    return Py_TYPE(o) == (PyTypeObject *)g_kv && plain_attr(o, s_length, false) && plain_attr(o, s_start, true);
}
bool plain_kv8(PyObject *o) { return Py_TYPE(o) == (PyTypeObject *)g_kv8 && plain_attr(o, s_length, false); }
bool plain_tensors(PyObject *const *a, std::initializer_list<int> at) {
    for (int i : at)
        if (!THPVariable_CheckExact(a[i])) return false;
    return true;
}
bool plain_kv4(PyObject *o) { return Py_TYPE(o) == (PyTypeObject *)g_kv4 && plain_attr(o, s_length, false); }
#define ORDINARY(n_args, cond) \
    if (n != (n_args) || !(cond)) Py_RETURN_NONE

struct View {
    mad_kv_view c;
    int32_t len[MAD_MAX_BATCH], start[MAD_MAX_BATCH];
    // KV `o` for B rows of [Hkv, cap, d] (Hkv < 0: any, returned in Hkv)
    mad_kv_view *read(PyObject *o, int B, int64_t *Hkv, int64_t d, const at::Tensor &like) {
        need(Py_TYPE(o) == (PyTypeObject *)g_kv && B <= MAD_MAX_BATCH);
        Ref ko(PyObject_GetAttr(o, s_k)), vo(PyObject_GetAttr(o, s_v)), lo(PyObject_GetAttr(o, s_length)),
            so(PyObject_GetAttr(o, s_start));
        const at::Tensor &k = tensor(ko.p), &v = tensor(vo.p);
        need(k.dim() == 4 && k.sizes() == v.sizes() && k.strides() == v.strides());
        need(k.stride(3) == 1 && k.stride(2) == k.size(3));
        need(k.size(0) == 1 || k.size(0) == B);
        if (*Hkv < 0) *Hkv = k.size(1);
        need(k.size(1) == *Hkv && k.size(3) == d);
        need(k.scalar_type() == like.scalar_type() && v.scalar_type() == like.scalar_type());
        need(k.device() == like.device() && v.device() == like.device());
        ints(lo.p, B, len);
        if (so.p != Py_None) ints(so.p, B, start);
        c.k = k.data_ptr();
        c.v = v.data_ptr();
        c.seq_stride = k.size(0) > 1 ? k.stride(0) : 0;
        c.head_stride = k.stride(1);
        c.cap = small(k.size(2));
        c.start = so.p != Py_None ? start : nullptr;
        c.len = len;
        return &c;
    }
};

struct View8 {
    mad_kv8_view c;
    int32_t len[MAD_MAX_BATCH];
    // KV8 `o` for B rows of [Hkv, cap, d] (Hkv < 0: any, returned in Hkv)
    mad_kv8_view *read(PyObject *o, int B, int64_t *Hkv, int64_t d, const at::Device &dev) {
        need(Py_TYPE(o) == (PyTypeObject *)g_kv8 && B >= 1 && B <= MAD_MAX_BATCH);
        Ref ko(PyObject_GetAttr(o, s_k)), vo(PyObject_GetAttr(o, s_v)), kso(PyObject_GetAttr(o, s_k_scale)),
            vso(PyObject_GetAttr(o, s_v_scale)), lo(PyObject_GetAttr(o, s_length)), bo(PyObject_GetAttr(o, s_block));
        const at::Tensor &k = tensor(ko.p), &v = tensor(vo.p), &ks = tensor(kso.p), &vs = tensor(vso.p);
        need(k.dim() == 4 && k.sizes() == v.sizes() && k.strides() == v.strides());
        need(k.scalar_type() == at::kFloat8_e4m3fn && v.scalar_type() == at::kFloat8_e4m3fn);
        need(k.stride(3) == 1 && k.stride(2) == k.size(3));
        need(k.size(0) == 1 || k.size(0) == B);
        if (*Hkv < 0) *Hkv = k.size(1);
        need(k.size(1) == *Hkv && k.size(3) == d);
        c.block = as_int(bo.p);
        need(c.block == 16 || c.block == 32 || c.block == 64 || c.block == 128);
        c.cap = small(k.size(2));
        need(ks.dim() == 3 && shape(ks, {k.size(0), *Hkv, ((int64_t)c.cap + c.block - 1) / c.block}) && vs.sizes() == ks.sizes());
        need(ks.strides() == vs.strides() && ks.stride(2) == 1 && ks.scalar_type() == at::kFloat && vs.scalar_type() == at::kFloat);
        need(k.device() == dev && v.device() == dev && ks.device() == dev && vs.device() == dev);
        ints(lo.p, B, len);
        const bool many = k.size(0) > 1;
        c.k = k.data_ptr();
        c.v = v.data_ptr();
        c.k_scale = (float *)ks.data_ptr();
        c.v_scale = (float *)vs.data_ptr();
        c.seq_stride = many ? k.stride(0) : 0;
        c.head_stride = k.stride(1);
        c.scale_seq_stride = many ? ks.stride(0) : 0;
        c.scale_head_stride = ks.stride(1);
        c.len = len;
        return &c;
    }
};

struct View4 {
    mad_kv4_view c;
    int32_t len[MAD_MAX_BATCH];
    // KV4 `o` for B rows of [Hkv, cap, d] (Hkv < 0: any, returned in Hkv)
    mad_kv4_view *read(PyObject *o, int B, int64_t *Hkv, int64_t d, const at::Device &dev) {
        need(Py_TYPE(o) == (PyTypeObject *)g_kv4 && B >= 1 && B <= MAD_MAX_BATCH);
        Ref ko(PyObject_GetAttr(o, s_k)), vo(PyObject_GetAttr(o, s_v)), kso(PyObject_GetAttr(o, s_k_scale)),
            vso(PyObject_GetAttr(o, s_v_scale)), lo(PyObject_GetAttr(o, s_length));
        const at::Tensor &k = tensor(ko.p), &v = tensor(vo.p), &ks = tensor(kso.p), &vs = tensor(vso.p);
        need(k.dim() == 4 && k.sizes() == v.sizes() && k.strides() == v.strides());
        need(k.scalar_type() == at::kByte && v.scalar_type() == at::kByte && ks.scalar_type() == at::kByte && vs.scalar_type() == at::kByte);
        need(k.stride(3) == 1 && k.stride(2) == k.size(3));
        need(k.size(0) == 1 || k.size(0) == B);
        if (*Hkv < 0) *Hkv = k.size(1);
        need(k.size(1) == *Hkv && 2 * k.size(3) == d);
        c.cap = small(k.size(2));
        need(shape(ks, {k.size(0), *Hkv, c.cap, d / 32}) && vs.sizes() == ks.sizes() && ks.strides() == vs.strides());
        need(ks.stride(3) == 1 && ks.stride(2) == d / 32);
        need(k.device() == dev && v.device() == dev && ks.device() == dev && vs.device() == dev);
        ints(lo.p, B, len);
        const bool many = k.size(0) > 1;
        c.k = k.data_ptr();
        c.v = v.data_ptr();
        c.k_scale = ks.data_ptr();
        c.v_scale = vs.data_ptr();
        c.seq_stride = many ? k.stride(0) : 0;
        c.head_stride = k.stride(1);
        c.scale_seq_stride = many ? ks.stride(0) : 0;
        c.scale_head_stride = ks.stride(1);
        c.len = len;
        return &c;
    }
};

// rows of heads [B, n_cap, H, d] whose heads lie one after the other
mad_rows rows_of(const at::Tensor &t, const at::Device &dev) {
    need(t.dim() == 4 && t.device() == dev && t.is_cuda() && t.layout() == at::kStrided && t.stride(3) == 1 &&
         (t.size(2) == 1 || t.stride(2) == t.size(3)));
    return {t.data_ptr(), t.stride(0), t.stride(1)};
}

void *stream_of(const at::Device &dev) {
    Ref index(PyLong_FromLong(dev.index()));
    Ref s(PyObject_CallOneArg(g_stream, index.p));
    void *p = PyLong_AsVoidPtr(s.p);
    need(!PyErr_Occurred());
    return p;
}

// the caller's workspace, or the one kept for (device, stream) if it is large enough.  It is held until the C entry
// point has returned: without the interpreter lock another thread may put a larger one in the kept one's place, and
// memory given back before this call's kernels are enqueued could be another tensor's by the time they run.
struct Scratch {
    const Ref held;
    void *p;
    size_t n;
    Scratch(PyObject *ws, const at::Device &dev, void *stream, size_t bytes) : held(of(ws, dev, stream)) {
        const at::Tensor &t = tensor(held.p);
        need((size_t)t.numel() >= bytes);
        p = t.data_ptr();
        n = (size_t)t.numel();
    }
    static PyObject *of(PyObject *ws, const at::Device &dev, void *stream) {   // an owned reference
        if (ws != Py_None) {
            Py_INCREF(ws);
            return ws;
        }
        Ref key(Py_BuildValue("(iN)", (int)dev.index(), PyLong_FromVoidPtr(stream)));
        PyObject *w = PyDict_GetItemWithError(g_ws, key.p);
        need(w != nullptr);
        return PyObject_GetAttr(w, s_buf);
    }
};

template <typename F> PyObject *guarded(F f) {
    try {
        return PyLong_FromLong(f());
    } catch (...) {   // Unhandled, or a C++ error of a tensor accessor
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}
// The call, on the device of its tensors: each has a default stream of its own, and a launch on it goes to the current
// device.  (Nothing to look up where the process sees one device: 0.2 us of a call's 4.)
bool several_devices() {
    static const bool several = c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).deviceCount() > 1;
    return several;
}
#define RELEASED(call)                                     \
    c10::OptionalDeviceGuard on_device;                    \
    if (several_devices()) on_device.reset_device(dev);    \
    int rc;                                                \
    Py_BEGIN_ALLOW_THREADS                                 \
    rc = (call);                                           \
    Py_END_ALLOW_THREADS                                   \
    return rc

float scale_of(PyObject *o, int64_t d) { return o == Py_None ? (float)std::pow((double)d, -0.5) : (float)as_double(o); }

// attn(q, mem, win, k_new, v_new, out, lse, scale, ws, modes | None)
PyObject *attn(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(10, plain_tensors(a, {0, 5, 6}) && (a[1] == Py_None || plain_kv(a[1])) && (a[2] == Py_None || plain_kv(a[2])) &&
                     (a[1] != Py_None || a[2] != Py_None) && (a[7] == Py_None || plain_real(a[7])) &&
                     (a[9] == Py_None || plain_ints(a[9])));
    return guarded([&]() -> int {
        const at::Tensor &q = first(a[0]);
        const at::Device dev = q.device();
        need(q.dim() == 3);
        const int B = small(q.size(0)), Hq = small(q.size(1)), d = small(q.size(2));
        int64_t Hkv = -1;
        View mem, win;
        mad_kv_view *mv = a[1] != Py_None ? mem.read(a[1], B, &Hkv, d, q) : nullptr;
        mad_kv_view *wv = a[2] != Py_None ? win.read(a[2], B, &Hkv, d, q) : nullptr;
        need(Hkv >= 1 && Hq % Hkv == 0);
        const at::Tensor &out = dense(a[5], dev), &lse = dense(a[6], dev);
        need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type());
        need(shape(lse, {B, Hq}) && lse.scalar_type() == at::kFloat);
        need((a[3] == Py_None) == (a[4] == Py_None));
        void *kn = nullptr, *vn = nullptr;
        if (a[3] != Py_None) {
            const at::Tensor &k = dense(a[3], dev), &v = dense(a[4], dev);
            need(shape(k, {B, Hkv, d}) && shape(v, {B, Hkv, d}) && k.scalar_type() == q.scalar_type() &&
                 v.scalar_type() == q.scalar_type());
            kn = k.data_ptr();
            vn = v.data_ptr();
        }
        const float scale = scale_of(a[7], d);
        uint8_t modes[MAD_MAX_BATCH];
        const bool step = a[9] != Py_None;
        if (step) ints(a[9], B, modes);
        void *st = stream_of(dev);
        const Scratch ws(a[8], dev, st, g.ws_bytes(MAD_OP_DECODE, B, Hq, (int)Hkv, d, 1, 0));
        const int dt = dtype_code(q);
        void *qp = q.data_ptr(), *op = out.data_ptr();
        float *lp = (float *)lse.data_ptr();
        if (step) {
            RELEASED(g.step(qp, B, Hq, (int)Hkv, d, dt, scale, mv, wv, kn, vn, modes, op, lp, ws.p, ws.n, st));
        }
        RELEASED(g.decode(qp, B, Hq, (int)Hkv, d, dt, scale, mv, wv, kn, vn, op, lp, ws.p, ws.n, st));
    });
}

// update(x, w_kv, pos, mem, fire | None, rope_base)
PyObject *update(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(6, plain_tensors(a, {0, 1}) && plain_rows(a[2]) && plain_kv(a[3]) && plain_flags(a[4]) && plain_real(a[5]));
    return guarded([&]() -> int {
        const at::Tensor &x = first(a[0]);
        const at::Device dev = x.device();
        const at::Tensor &w = dense(a[1], dev);
        need(x.dim() == 3);
        const int B = small(x.size(0)), nn = small(x.size(1)), D = small(x.size(2));
        need(B <= MAD_MAX_BATCH && (int64_t)B * nn <= MAD_MAX_UPDATE_ROWS && w.dim() == 2 && w.size(1) == D &&
             w.scalar_type() == x.scalar_type());
        Ref ko(PyObject_GetAttr(a[3], s_k));
        const at::Tensor &k = tensor(ko.p);
        need(k.dim() == 4);
        int64_t Hkv = k.size(1);
        const int d = small(k.size(3));
        need(w.size(0) == 2 * Hkv * d);
        View mem;
        mad_kv_view *mv = mem.read(a[3], B, &Hkv, d, x);
        need((PyList_CheckExact(a[2]) || PyTuple_CheckExact(a[2])) && PySequence_Fast_GET_SIZE(a[2]) == B);
        int32_t pos[MAD_MAX_UPDATE_ROWS];
        for (int b = 0; b < B; ++b) ints(PySequence_Fast_ITEMS(a[2])[b], nn, pos + (size_t)b * nn);
        uint8_t fire[MAD_MAX_BATCH];
        if (a[4] != Py_None) {
            need((PyList_CheckExact(a[4]) || PyTuple_CheckExact(a[4])) && PySequence_Fast_GET_SIZE(a[4]) == B);
            for (int b = 0; b < B; ++b) {
                PyObject *f = PySequence_Fast_ITEMS(a[4])[b];
                need(PyBool_Check(f) || PyLong_CheckExact(f));
                fire[b] = PyObject_IsTrue(f) ? 1 : 0;
            }
        }
        const double base = as_double(a[5]);
        const int dt = dtype_code(x);
        void *st = stream_of(dev), *xp = x.data_ptr(), *wp = w.data_ptr();
        const uint8_t *fp = a[4] != Py_None ? fire : nullptr;
        RELEASED(g.update(xp, wp, pos, fp, B, nn, D, (int)Hkv, d, dt, base, mv, st));
    });
}

// verify(q, kv, out, lse, scale, ws)
PyObject *verify(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(6, plain_tensors(a, {0, 2, 3}) && plain_kv(a[1]) && (a[4] == Py_None || plain_real(a[4])));
    return guarded([&]() -> int {
        const at::Tensor &q = first(a[0]);
        const at::Device dev = q.device();
        need(q.dim() == 4);
        const int B = small(q.size(0)), T = small(q.size(1)), Hq = small(q.size(2)), d = small(q.size(3));
        int64_t Hkv = -1;
        View kv;
        mad_kv_view *v = kv.read(a[1], B, &Hkv, d, q);
        need(v->start == nullptr && Hkv >= 1);
        const at::Tensor &out = dense(a[2], dev), &lse = dense(a[3], dev);
        need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type());
        need(shape(lse, {B, T, Hq}) && lse.scalar_type() == at::kFloat);
        const float scale = scale_of(a[4], d);
        void *st = stream_of(dev);
        const Scratch ws(a[5], dev, st, g.ws_bytes(MAD_OP_VERIFY, B, Hq, (int)Hkv, d, T, 0));
        const int dt = dtype_code(q);
        void *qp = q.data_ptr(), *op = out.data_ptr();
        float *lp = (float *)lse.data_ptr();
        RELEASED(g.verify(qp, B, T, Hq, (int)Hkv, d, dt, scale, v, op, lp, ws.p, ws.n, st));
    });
}

// verify_vt(q, k, vt, length, out, lse, scale, ws)
PyObject *verify_vt(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(8, plain_tensors(a, {0, 1, 2, 4, 5}) && plain_ints(a[3]) && (a[6] == Py_None || plain_real(a[6])));
    return guarded([&]() -> int {
        const at::Tensor &q = first(a[0]);
        const at::Device dev = q.device();
        const at::Tensor &k = tensor(a[1]), &vt = tensor(a[2]);
        need(q.dim() == 4 && k.dim() == 4 && vt.dim() == 4);
        const int B = small(q.size(0)), T = small(q.size(1)), Hq = small(q.size(2)), d = small(q.size(3));
        const int Hkv = small(k.size(1)), cap = small(k.size(2));
        need(B <= MAD_MAX_BATCH && shape(vt, {B, Hkv, d, cap}) && shape(k, {B, Hkv, cap, d}));
        need(k.stride(3) == 1 && k.stride(2) == d && vt.stride(3) == 1 && vt.stride(2) == cap);
        need(k.stride(0) == vt.stride(0) && k.stride(1) == vt.stride(1));
        need(k.scalar_type() == q.scalar_type() && vt.scalar_type() == q.scalar_type() && k.device() == dev && vt.device() == dev);
        int32_t len[MAD_MAX_BATCH];
        ints(a[3], B, len);
        const at::Tensor &out = dense(a[4], dev), &lse = dense(a[5], dev);
        need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type());
        need(shape(lse, {B, T, Hq}) && lse.scalar_type() == at::kFloat);
        const float scale = scale_of(a[6], d);
        void *st = stream_of(dev);
        const Scratch ws(a[7], dev, st, g.ws_bytes(MAD_OP_VERIFY, B, Hq, Hkv, d, T, 0));
        const int dt = dtype_code(q);
        void *qp = q.data_ptr(), *op = out.data_ptr(), *kp = k.data_ptr(), *vp = vt.data_ptr();
        float *lp = (float *)lse.data_ptr();
        const int64_t seq = B > 1 ? k.stride(0) : 0, head = k.stride(1);
        RELEASED(g.verify_vt(qp, B, T, Hq, Hkv, d, dt, scale, kp, vp, seq, head, cap, len, op, lp, ws.p, ws.n, st));
    });
}

// kv8_append(k_new, v_new, kv, n | None)
PyObject *kv8_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(4, plain_tensors(a, {0, 1}) && plain_kv8(a[2]) && (a[3] == Py_None || plain_ints(a[3])));
    return guarded([&]() -> int {
        const at::Tensor &k = first(a[0]);
        const at::Device dev = k.device();
        const at::Tensor &v = dense(a[1], dev);
        need(k.dim() == 4 && v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type());
        const int B = small(k.size(0)), n_cap = small(k.size(1)), d = small(k.size(3));
        int64_t Hkv = small(k.size(2));
        View8 kv;
        mad_kv8_view *c = kv.read(a[2], B, &Hkv, d, dev);
        int32_t rows[MAD_MAX_BATCH];
        if (a[3] != Py_None) ints(a[3], B, rows);
        const int32_t *np = a[3] != Py_None ? rows : nullptr;
        const int dt = dtype_code(k);
        void *st = stream_of(dev), *kp = k.data_ptr(), *vp = v.data_ptr();
        RELEASED(g.kv8_append(kp, vp, np, B, n_cap, (int)Hkv, d, dt, c, st));
    });
}

// verify8(q, kv, out, lse, scale, ws)
PyObject *verify8(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(6, plain_tensors(a, {0, 2, 3}) && plain_kv8(a[1]) && (a[4] == Py_None || plain_real(a[4])));
    return guarded([&]() -> int {
        const at::Tensor &q = first(a[0]);
        const at::Device dev = q.device();
        need(q.dim() == 4);
        const int B = small(q.size(0)), T = small(q.size(1)), Hq = small(q.size(2)), d = small(q.size(3));
        int64_t Hkv = -1;
        View8 kv;
        mad_kv8_view *v = kv.read(a[1], B, &Hkv, d, dev);
        need(Hkv >= 1 && Hq % Hkv == 0);
        const at::Tensor &out = dense(a[2], dev), &lse = dense(a[3], dev);
        need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type());
        need(shape(lse, {B, T, Hq}) && lse.scalar_type() == at::kFloat);
        const float scale = scale_of(a[4], d);
        void *st = stream_of(dev);
        const Scratch ws(a[5], dev, st, g.ws_bytes(MAD_OP_VERIFY, B, Hq, (int)Hkv, d, T, 0));
        const int dt = dtype_code(q);
        void *qp = q.data_ptr(), *op = out.data_ptr();
        float *lp = (float *)lse.data_ptr();
        RELEASED(g.verify8(qp, B, T, Hq, (int)Hkv, d, dt, scale, v, op, lp, ws.p, ws.n, st));
    });
}

const at::Tensor &i32(PyObject *o, const at::Device &dev, std::initializer_list<int64_t> want) {
    const at::Tensor &t = dense(o, dev);
    need(t.scalar_type() == at::kInt && shape(t, want));
    return t;
}

// greedy(logits, draft | None, n_accept, next_tok, ws)
PyObject *greedy(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(5, plain_tensors(a, {0, 2, 3}) && (a[1] == Py_None || THPVariable_CheckExact(a[1])));
    return guarded([&]() -> int {
        const at::Tensor &x = first(a[0]);
        const at::Device dev = x.device();
        need(x.dim() == 3);
        const int B = small(x.size(0)), T = small(x.size(1)), V = small(x.size(2));
        int32_t *draft = T > 1 ? (int32_t *)i32(a[1], dev, {B, T - 1}).data_ptr() : nullptr;
        need(T > 1 || a[1] == Py_None);
        int32_t *na = (int32_t *)i32(a[2], dev, {B}).data_ptr(), *nt = (int32_t *)i32(a[3], dev, {B}).data_ptr();
        void *st = stream_of(dev);
        const Scratch ws(a[4], dev, st, g.ws_bytes(MAD_OP_ACCEPT, B, 1, 1, 64, T, V));
        const int dt = dtype_code(x);
        void *xp = x.data_ptr();
        RELEASED(g.greedy(xp, dt, draft, B, T, V, na, nt, ws.p, ws.n, st));
    });
}

// a number for all of n sequences, or a list or tuple of them
bool plain_reals(PyObject *o) {
    if (plain_real(o)) return true;
    const Py_ssize_t n = PyList_CheckExact(o) || PyTuple_CheckExact(o) ? PySequence_Fast_GET_SIZE(o) : 0;
    return n > 0 && plain_real(PySequence_Fast_GET_ITEM(o, 0)) && plain_real(PySequence_Fast_GET_ITEM(o, n - 1));
}
void reals(PyObject *o, int n, double *out) {
    if (plain_real(o)) {
        const double v = as_double(o);
        for (int i = 0; i < n; ++i) out[i] = v;
        return;
    }
    need(PySequence_Fast_GET_SIZE(o) == n);
    for (int i = 0; i < n; ++i) {
        PyObject *x = PySequence_Fast_ITEMS(o)[i];
        need(plain_real(x));
        out[i] = as_double(x);
    }
}

// sample(logits, u | None, temperature, top_k, top_p, min_p, tok | None, probs | None, ws)
PyObject *sample(PyObject *, PyObject *const *a, Py_ssize_t n) {
    auto maybe = [&](int i) { return a[i] == Py_None || THPVariable_CheckExact(a[i]); };
    ORDINARY(9, plain_tensors(a, {0}) && maybe(1) && maybe(6) && maybe(7) && plain_reals(a[2]) &&
                    (PyLong_CheckExact(a[3]) || plain_ints(a[3])) && plain_reals(a[4]) && plain_reals(a[5]));
    return guarded([&]() -> int {
        const at::Tensor &x = first(a[0]);
        const at::Device dev = x.device();
        need(x.dim() == 3);
        const int B = small(x.size(0)), T = small(x.size(1)), V = small(x.size(2));
        need(B >= 1 && B <= MAD_MAX_BATCH);
        double t[MAD_MAX_BATCH], p[MAD_MAX_BATCH], mp[MAD_MAX_BATCH];
        int32_t k[MAD_MAX_BATCH];
        reals(a[2], B, t);
        reals(a[4], B, p);
        reals(a[5], B, mp);
        if (PyLong_CheckExact(a[3])) {
            const int v = as_int(a[3]);
            for (int b = 0; b < B; ++b) k[b] = v;
        } else {
            ints(a[3], B, k);
        }
        const float *u = nullptr;
        int32_t *tok = nullptr;
        float *probs = nullptr;
        if (a[1] != Py_None) {
            const at::Tensor &w = dense(a[1], dev);
            need(shape(w, {B, T}) && w.scalar_type() == at::kFloat);
            u = (const float *)w.data_ptr();
        }
        if (a[6] != Py_None) tok = (int32_t *)i32(a[6], dev, {B, T}).data_ptr();
        if (a[7] != Py_None) {
            const at::Tensor &w = dense(a[7], dev);
            need(shape(w, {B, T, V}) && w.scalar_type() == at::kFloat);
            probs = (float *)w.data_ptr();
        }
        need((tok || probs) && (u || !tok) && (tok || !u));
        void *st = stream_of(dev);
        const Scratch ws(a[8], dev, st, g.ws_bytes(MAD_OP_SAMPLE, B, 1, 1, 64, T, V));
        const int dt = dtype_code(x);
        void *xp = x.data_ptr();
        RELEASED(g.sample(xp, dt, u, t, k, p, mp, B, T, V, tok, probs, ws.p, ws.n, st));
    });
}

// qk_norm_rope(q | None, k | None, pos, q_gamma | None, k_gamma | None, q_out, k_out, n | None, eps, rope_base | None)
PyObject *qk_norm_rope(PyObject *, PyObject *const *a, Py_ssize_t n) {
    auto maybe = [&](int i) { return a[i] == Py_None || THPVariable_CheckExact(a[i]); };
    ORDINARY(10, maybe(0) && maybe(1) && (a[0] != Py_None || a[1] != Py_None) && maybe(3) && maybe(4) &&
                     (a[5] != Py_None || a[0] == Py_None) && (a[6] != Py_None || a[1] == Py_None) && maybe(5) && maybe(6) &&
                     (a[7] == Py_None || plain_ints(a[7])) && plain_real(a[8]) && (a[9] == Py_None || plain_real(a[9])) &&
                     (a[9] == Py_None || plain_ints(a[2]) || THPVariable_CheckExact(a[2])));
    return guarded([&]() -> int {
        const at::Tensor &like = tensor(a[0] != Py_None ? a[0] : a[1]);
        const at::Device dev = like.device();
        need(like.dim() == 4);
        const int B = small(like.size(0)), n_cap = small(like.size(1)), d = small(like.size(3));
        need(B >= 1 && B <= MAD_MAX_BATCH);
        mad_rows in[2], out[2];
        void *gamma[2] = {nullptr, nullptr};
        int heads[2] = {0, 0};
        for (int i = 0; i < 2; ++i) {
            if (a[i] == Py_None) {
                need(a[3 + i] == Py_None && a[5 + i] == Py_None);
                continue;
            }
            const at::Tensor &x = tensor(a[i]), &y = tensor(a[5 + i]);
            in[i] = rows_of(x, dev);
            out[i] = rows_of(y, dev);
            heads[i] = small(x.size(2));
            need(x.size(0) == B && x.size(1) == n_cap && x.size(3) == d && x.scalar_type() == like.scalar_type());
            need(y.sizes() == x.sizes() && y.scalar_type() == x.scalar_type());
            if (a[3 + i] != Py_None) {
                const at::Tensor &gm = dense(a[3 + i], dev);
                need(shape(gm, {d}) && gm.scalar_type() == like.scalar_type());
                gamma[i] = gm.data_ptr();
            }
        }
        int32_t start[MAD_MAX_BATCH], rows[MAD_MAX_BATCH];
        const int32_t *sp = nullptr, *pp = nullptr, *np = nullptr;
        double base = 0.0;
        if (a[9] != Py_None) {
            base = as_double(a[9]);
            if (THPVariable_CheckExact(a[2])) {
                const at::Tensor &p = dense(a[2], dev);
                need(shape(p, {B, n_cap}) && p.scalar_type() == at::kInt);
                pp = (const int32_t *)p.data_ptr();
            } else {
                ints(a[2], B, start);
                sp = start;
            }
        }
        if (a[7] != Py_None) {
            ints(a[7], B, rows);
            np = rows;
        }
        const float eps = (float)as_double(a[8]);
        const int dt = dtype_code(like);
        void *st = stream_of(dev);
        const bool q = a[0] != Py_None, k = a[1] != Py_None;
        RELEASED(g.norm_rope(q ? &in[0] : nullptr, k ? &in[1] : nullptr, q ? &out[0] : nullptr, k ? &out[1] : nullptr, gamma[0], gamma[1],
                             eps, base, sp, pp, np, B, n_cap, heads[0], heads[1], d, dt, st));
    });
}

// kv4_append(k_new, v_new, kv, n | None, k_held | None, v_held | None)
PyObject *kv4_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(6, plain_tensors(a, {0, 1}) && plain_kv4(a[2]) && (a[3] == Py_None || plain_ints(a[3])) &&
                    ((a[4] == Py_None && a[5] == Py_None) || plain_tensors(a, {4, 5})));
    return guarded([&]() -> int {
        const at::Tensor &k = tensor(a[0]), &v = tensor(a[1]);
        const at::Device dev = k.device();
        mad_rows r[4] = {rows_of(k, dev), rows_of(v, dev)};
        need(v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type());
        const bool held = a[4] != Py_None;
        for (int i = 2; held && i < 4; ++i) {
            const at::Tensor &t = tensor(a[2 + i]);
            need(t.sizes() == k.sizes() && t.scalar_type() == k.scalar_type());
            r[i] = rows_of(t, dev);
        }
        const int B = small(k.size(0)), n_cap = small(k.size(1)), d = small(k.size(3));
        int64_t Hkv = small(k.size(2));
        View4 kv;
        mad_kv4_view *c = kv.read(a[2], B, &Hkv, d, dev);
        int32_t rows[MAD_MAX_BATCH];
        if (a[3] != Py_None) ints(a[3], B, rows);
        const int32_t *np = a[3] != Py_None ? rows : nullptr;
        const int dt = dtype_code(k);
        void *st = stream_of(dev);
        RELEASED(g.kv4_append(&r[0], &r[1], held ? &r[2] : nullptr, held ? &r[3] : nullptr, np, B, n_cap, (int)Hkv, d, dt, c, st));
    });
}

// verify4(q, kv, out, lse, scale, ws)
PyObject *verify4(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(6, plain_tensors(a, {0, 2, 3}) && plain_kv4(a[1]) && (a[4] == Py_None || plain_real(a[4])));
    return guarded([&]() -> int {
        const at::Tensor &q = first(a[0]);
        const at::Device dev = q.device();
        need(q.dim() == 4);
        const int B = small(q.size(0)), T = small(q.size(1)), Hq = small(q.size(2)), d = small(q.size(3));
        int64_t Hkv = -1;
        View4 kv;
        mad_kv4_view *v = kv.read(a[1], B, &Hkv, d, dev);
        need(Hkv >= 1 && Hq % Hkv == 0);
        const at::Tensor &out = dense(a[2], dev), &lse = dense(a[3], dev);
        need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type());
        need(shape(lse, {B, T, Hq}) && lse.scalar_type() == at::kFloat);
        const float scale = scale_of(a[4], d);
        void *st = stream_of(dev);
        const Scratch ws(a[5], dev, st, g.ws_bytes(MAD_OP_VERIFY_KV4, B, Hq, (int)Hkv, d, T, 0));
        const int dt = dtype_code(q);
        void *qp = q.data_ptr(), *op = out.data_ptr();
        float *lp = (float *)lse.data_ptr();
        RELEASED(g.verify4(qp, B, T, Hq, (int)Hkv, d, dt, scale, v, op, lp, ws.p, ws.n, st));
    });
}

// logprobs(logits, tok | None, top_n, temperature, logp, rank, entropy, top_tok, top_logp, ws): every output there is given
PyObject *logprobs(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(10, plain_tensors(a, {0, 6}) && PyLong_CheckExact(a[2]) && plain_reals(a[3]) &&
                     (a[1] == Py_None ? a[4] == Py_None && a[5] == Py_None : plain_tensors(a, {1, 4, 5})) &&
                     ((a[7] == Py_None && a[8] == Py_None) || plain_tensors(a, {7, 8})));
    return guarded([&]() -> int {
        const at::Tensor &x = tensor(a[0]);
        const at::Device dev = x.device();
        need(x.dim() == 3 && x.is_cuda() && x.layout() == at::kStrided);
        const int B = small(x.size(0)), T = small(x.size(1)), V = small(x.size(2)), top = as_int(a[2]);
        need(B >= 1 && B <= MAD_MAX_BATCH && (V == 1 || x.stride(2) == 1));
        need(top >= 0 && top <= MAD_MAX_TOP && top <= V && (top > 0) == (a[7] != Py_None));
        double temp[MAD_MAX_BATCH];
        reals(a[3], B, temp);
        auto f32 = [&](PyObject *o, std::initializer_list<int64_t> want) {
            const at::Tensor &t = dense(o, dev);
            need(shape(t, want) && t.scalar_type() == at::kFloat);
            return (float *)t.data_ptr();
        };
        const int32_t *tok = nullptr;
        float *lp = nullptr, *ent = f32(a[6], {B, T}), *tl = nullptr;
        int32_t *rank = nullptr, *tt = nullptr;
        if (a[1] != Py_None) {
            tok = (const int32_t *)i32(a[1], dev, {B, T}).data_ptr();
            lp = f32(a[4], {B, T});
            rank = (int32_t *)i32(a[5], dev, {B, T}).data_ptr();
        }
        if (top > 0) {
            tt = (int32_t *)i32(a[7], dev, {B, T, top}).data_ptr();
            tl = f32(a[8], {B, T, top});
        }
        void *st = stream_of(dev);
        const Scratch ws(a[9], dev, st, g.ws_bytes(MAD_OP_LOGPROBS, B, 1, 1, 64, T, V));
        const int dt = dtype_code(x);
        void *xp = x.data_ptr();
        const int64_t seq = x.stride(0), row = x.stride(1);
        RELEASED(g.logprobs(xp, dt, seq, row, tok, temp, B, T, V, top, lp, rank, ent, tt, tl, ws.p, ws.n, st));
    });
}

// stoch(p, q, draft, u, n_accept, next_tok, ws)
PyObject *stoch(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(7, plain_tensors(a, {0, 1, 2, 3, 4, 5}));
    return guarded([&]() -> int {
        const at::Tensor &p = first(a[0]);
        const at::Device dev = p.device();
        need(p.dim() == 3 && p.scalar_type() == at::kFloat);
        const int B = small(p.size(0)), T = small(p.size(1)), V = small(p.size(2));
        need(T > 1);
        const at::Tensor &q = dense(a[1], dev), &u = dense(a[3], dev);
        need(shape(q, {B, T - 1, V}) && q.scalar_type() == at::kFloat && shape(u, {B, T}) && u.scalar_type() == at::kFloat);
        int32_t *draft = (int32_t *)i32(a[2], dev, {B, T - 1}).data_ptr();
        int32_t *na = (int32_t *)i32(a[4], dev, {B}).data_ptr(), *nt = (int32_t *)i32(a[5], dev, {B}).data_ptr();
        void *st = stream_of(dev);
        const Scratch ws(a[6], dev, st, g.ws_bytes(MAD_OP_ACCEPT_STOCH, B, 1, 1, 64, T, V));
        const float *pp = (const float *)p.data_ptr(), *qp = (const float *)q.data_ptr(), *up = (const float *)u.data_ptr();
        RELEASED(g.stoch(pp, qp, draft, up, B, T, V, na, nt, ws.p, ws.n, st));
    });
}

// qkv(x, gamma, w, pos, Hq, Hkv, d, q, k, v, xn | None, eps, rope_base, kv_from_row0)
PyObject *qkv(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(14, plain_tensors(a, {0, 1, 2, 7, 8, 9}) && plain_ints(a[3]) && plain_real(a[11]) && plain_real(a[12]) &&
                     PyBool_Check(a[13]));
    return guarded([&]() -> int {
        const at::Tensor &x = first(a[0]);
        const at::Device dev = x.device();
        need(x.dim() == 2 && x.scalar_type() == at::kBFloat16);
        const int R = small(x.size(0)), D = small(x.size(1)), Hq = as_int(a[4]), Hkv = as_int(a[5]), d = as_int(a[6]);
        need(R <= MAD_MAX_LAYER_ROWS);
        const at::Tensor &gm = dense(a[1], dev), &w = dense(a[2], dev), &q = dense(a[7], dev), &k = dense(a[8], dev),
                         &v = dense(a[9], dev);
        need(shape(gm, {D}) && shape(w, {((int64_t)Hq + 2 * Hkv) * d, D}) && shape(q, {R, Hq, d}) && shape(k, {R, Hkv, d}) &&
             shape(v, {R, Hkv, d}));
        void *xn = nullptr;
        if (a[10] != Py_None) {
            const at::Tensor &t = dense(a[10], dev);
            need(shape(t, {R, D}));
            xn = t.data_ptr();
        }
        int32_t pos[MAD_MAX_LAYER_ROWS];
        ints(a[3], R, pos);
        const float eps = (float)as_double(a[11]);
        const double base = as_double(a[12]);
        const int row0 = a[13] == Py_True;
        void *st = stream_of(dev), *xp = x.data_ptr(), *gp = gm.data_ptr(), *wp = w.data_ptr(), *qp = q.data_ptr(),
             *kp = k.data_ptr(), *vp = v.data_ptr();
        RELEASED(g.qkv(xp, gp, eps, wp, pos, R, D, Hq, Hkv, d, base, row0, qp, kp, vp, xn, st));
    });
}

// linear(x, w, res, out)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(4, plain_tensors(a, {0, 1, 2, 3}));
    return guarded([&]() -> int {
        const at::Tensor &x = first(a[0]);
        const at::Device dev = x.device();
        const at::Tensor &w = dense(a[1], dev), &res = dense(a[2], dev), &out = dense(a[3], dev);
        need(x.dim() == 2 && w.dim() == 2 && x.scalar_type() == at::kBFloat16);
        const int R = small(x.size(0)), D = small(x.size(1)), N = small(w.size(0));
        need(shape(w, {N, D}) && shape(res, {R, N}) && shape(out, {R, N}));
        void *st = stream_of(dev), *xp = x.data_ptr(), *wp = w.data_ptr(), *rp = res.data_ptr(), *op = out.data_ptr();
        RELEASED(g.linear(xp, wp, rp, R, D, N, op, st));
    });
}

// swiglu(x, gamma, w_gate_up, out, eps)
PyObject *swiglu(PyObject *, PyObject *const *a, Py_ssize_t n) {
    ORDINARY(5, plain_tensors(a, {0, 1, 2, 3}) && plain_real(a[4]));
    return guarded([&]() -> int {
        const at::Tensor &x = first(a[0]);
        const at::Device dev = x.device();
        const at::Tensor &gm = dense(a[1], dev), &w = dense(a[2], dev), &out = dense(a[3], dev);
        need(x.dim() == 2 && w.dim() == 2 && x.scalar_type() == at::kBFloat16);
        const int R = small(x.size(0)), D = small(x.size(1)), F = small(w.size(0) / 2);
        need(shape(gm, {D}) && shape(w, {2 * (int64_t)F, D}) && shape(out, {R, F}));
        const float eps = (float)as_double(a[4]);
        void *st = stream_of(dev), *xp = x.data_ptr(), *gp = gm.data_ptr(), *wp = w.data_ptr(), *op = out.data_ptr();
        RELEASED(g.swiglu(xp, gp, eps, wp, R, D, F, op, st));
    });
}

// bind(addresses of the C entry points in Entry's order, KV, the default workspaces, the raw-stream getter)
PyObject *bind(PyObject *, PyObject *args) {
    PyObject *addr, *kv, *ws, *st;
    if (!PyArg_ParseTuple(args, "O!OO!O", &PyTuple_Type, &addr, &kv, &PyDict_Type, &ws, &st)) return nullptr;
    void *f[sizeof(Entry) / sizeof(void *)];
    const Py_ssize_t n = sizeof(f) / sizeof(f[0]);
    if (PyTuple_GET_SIZE(addr) != n) {
        PyErr_SetString(PyExc_ValueError, "bind: wrong number of entry points");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        f[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addr, i));
        if (PyErr_Occurred()) return nullptr;
    }
    memcpy(&g, f, sizeof(g));
    Py_INCREF(kv);
    Py_INCREF(ws);
    Py_INCREF(st);
    Py_XSETREF(g_kv, kv);
    Py_XSETREF(g_ws, ws);
    Py_XSETREF(g_stream, st);
    Py_RETURN_NONE;
}

// bind_kv8(KV8)
PyObject *bind_kv8(PyObject *, PyObject *kv8) {
    Py_INCREF(kv8);
    Py_XSETREF(g_kv8, kv8);
    Py_RETURN_NONE;
}

// bind_kv4(KV4)
PyObject *bind_kv4(PyObject *, PyObject *kv4) {
    Py_INCREF(kv4);
    Py_XSETREF(g_kv4, kv4);
    Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr}, {"bind_kv8", bind_kv8, METH_O, nullptr},
                         {"bind_kv4", bind_kv4, METH_O, nullptr}, FAST(attn), FAST(update), FAST(verify), FAST(verify_vt),
                         FAST(greedy), FAST(stoch), FAST(qkv), FAST(linear), FAST(swiglu), FAST(kv8_append),
                         FAST(verify8), FAST(sample), FAST(qk_norm_rope), FAST(kv4_append), FAST(verify4), FAST(logprobs), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) {
    s_k = PyUnicode_InternFromString("k");
    s_v = PyUnicode_InternFromString("v");
    s_length = PyUnicode_InternFromString("length");
    s_start = PyUnicode_InternFromString("start");
    s_buf = PyUnicode_InternFromString("buf");
    s_k_scale = PyUnicode_InternFromString("k_scale");
    s_v_scale = PyUnicode_InternFromString("v_scale");
    s_block = PyUnicode_InternFromString("block");
    return PyModule_Create(&module);
}

// The calls of a layer and of a decode step, from Python objects to the C ABI without ctypes: reading a tensor's address, shape and
// strides and converting a dozen arguments there takes 3 to 5 us of Python a call, which is what the smallest layers and the decode
// steps over short caches last (a layer of 4 heads, n = 576: four calls, 32.7 us of host time; a decode step: 4.8 us around two
// launches).  A call takes plain torch.Tensor objects and plain numbers; for whatever else (a subclass, another dtype, a shape or
// stride that is not as expected, CUDA not initialised) it returns None before anything is launched, and the caller goes the general way,
// which handles it or says what is wrong.  Otherwise it returns the library's error code.  The GIL is released around the library call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <climits>
#include <cstring>

#include "zipvl.h"

namespace {

PyObject *s_data_ptr, *s_shape, *s_dtype, *s_stride, *s_numel, *s_is_contiguous, *s_hi_codes, *s_hi_params, *s_lo_codes, *s_lo_params, *s_K, *s_V,
    *s_len_hi, *s_len_lo, *s_cap_hi, *s_cap_lo, *s_d, *s_on_device;
PyObject *g_tensor, *g_f32, *g_bf16, *g_i32, *g_u8, *g_is_initialized, *g_get_device, *g_get_stream;

// An owned reference.
struct Ref {
    PyObject* p;
    explicit Ref(PyObject* o) : p(o) {}
    ~Ref() { Py_XDECREF(p); }
    Ref(const Ref&) = delete;
    Ref& operator=(const Ref&) = delete;
};

// The arguments of a call; `ok` falls to false at the first that is not as expected.
struct Args {
    PyObject* const* a;
    bool ok = true;

    PyObject* method(PyObject* self, PyObject* name) { return PyObject_VectorcallMethod(name, &self, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr); }
    bool tensor(PyObject* t) { return ok = ok && Py_TYPE(t) == (PyTypeObject*)g_tensor; }
    long long number(PyObject* o) {
        if (!ok || !o || !PyLong_CheckExact(o)) { ok = false; return 0; }
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) ok = false;
        return v;
    }
    int int32(PyObject* o) {
        const long long v = number(o);
        if (v < INT_MIN || v > INT_MAX) ok = false;
        return ok ? (int)v : 0;
    }
    double real(PyObject* o) {
        if (!ok || !(PyFloat_CheckExact(o) || PyLong_CheckExact(o))) { ok = false; return 0; }
        const double v = PyFloat_AsDouble(o);
        if (v == -1 && PyErr_Occurred()) ok = false;
        return v;
    }
    void* address(PyObject* t) {
        if (!tensor(t)) return nullptr;
        Ref r(method(t, s_data_ptr));
        if (!r.p) { ok = false; return nullptr; }
        void* v = PyLong_AsVoidPtr(r.p);
        if (!v && PyErr_Occurred()) ok = false;
        return v;
    }
    void* address_or_null(PyObject* t) { return t == Py_None ? nullptr : address(t); }
    size_t bytes(PyObject* t) {                              // of a workspace: its elements are taken for bytes, as everywhere
        if (!tensor(t)) return 0;
        Ref r(method(t, s_numel));
        if (!r.p) { ok = false; return 0; }
        return (size_t)number(r.p);
    }
    void dense(PyObject* t) {
        if (t == Py_None || !tensor(t)) return;
        Ref r(method(t, s_is_contiguous));
        if (r.p != Py_True) ok = false;
    }
    template <int N> void extents(PyObject* tuple, int64_t (&out)[N]) {
        if (!ok || !tuple || !PyTuple_Check(tuple) || PyTuple_GET_SIZE(tuple) != N) { ok = false; return; }
        for (int i = 0; i < N; ++i) out[i] = number(PyTuple_GET_ITEM(tuple, i));
    }
    template <int N> void shape(PyObject* t, int64_t (&out)[N]) {
        if (!tensor(t)) return;
        Ref r(PyObject_GetAttr(t, s_shape));
        extents(r.p, out);
    }
    void strides(PyObject* t, int64_t (&out)[3]) {           // of a [B, H, n, d] view with contiguous rows
        if (!tensor(t)) return;
        Ref r(method(t, s_stride));
        int64_t st[4] = {};
        extents(r.p, st);
        if (st[3] != 1) ok = false;
        for (int i = 0; i < 3; ++i) out[i] = st[i];
    }
    int dtype(PyObject* t) {
        if (!tensor(t)) return 0;
        Ref r(PyObject_GetAttr(t, s_dtype));
        if (r.p != g_f32 && r.p != g_bf16) ok = false;
        return r.p == g_bf16;
    }
    int32_t narrow(int64_t v) {
        if (v < INT_MIN || v > INT_MAX) ok = false;
        return (int32_t)v;
    }
    // dims of a layer; q may be NULL (its heads are then K's), and v
    zipvl_dims layer(PyObject* q, PyObject* k, PyObject* v) {
        zipvl_dims d = {};
        int64_t sq[4] = {}, sk[4] = {};
        shape(k, sk);
        if (q) shape(q, sq);
        const int64_t* ref = q ? sq : sk;
        d.B = narrow(ref[0]); d.n = narrow(ref[2]); d.d = narrow(ref[3]);
        d.Hq = narrow(ref[1]); d.Hkv = narrow(sk[1]);
        d.dtype = dtype(q ? q : k);
        if (q) strides(q, d.q_strides);
        strides(k, d.k_strides);
        if (v) strides(v, d.v_strides);
        return d;
    }
    zipvl_dims step(PyObject* B, PyObject* Hq, PyObject* Hkv, int64_t n, int64_t dim, int code) {
        zipvl_dims d = {};
        d.B = int32(B); d.Hq = int32(Hq); d.Hkv = int32(Hkv);
        d.n = narrow(n); d.d = narrow(dim); d.dtype = code;
        return d;
    }
    // The tensors of positions and pages, which have to be on the current device: an address, with the shape, the type and contiguity checked.
    long on = -2;                                            // the device of those seen so far
    void* placed(PyObject* t) {
        void* v = address(t);
        if (!ok) return nullptr;
        Ref r(method(t, s_on_device));
        const long at = r.p && PyLong_CheckExact(r.p) ? PyLong_AsLong(r.p) : -1;
        if (at < 0 || (on != -2 && on != at)) ok = false;
        on = at;
        return v;
    }
    void typed(PyObject* t, PyObject* dtype) {
        if (!tensor(t)) return;
        Ref r(PyObject_GetAttr(t, s_dtype));
        if (r.p != dtype) ok = false;
    }
    template <int N> void* array(PyObject* t, PyObject* dtype, const int64_t (&want)[N]) {
        int64_t s[N] = {};
        shape(t, s);
        for (int i = 0; i < N; ++i)
            if (s[i] != want[i]) ok = false;
        typed(t, dtype);
        dense(t);
        return placed(t);
    }
    template <int N> void* ints(PyObject* t, const int64_t (&want)[N]) { return array(t, g_i32, want); }
    template <int N> void* ints_or_null(PyObject* t, const int64_t (&want)[N]) { return t == Py_None ? nullptr : ints(t, want); }
    void* table(PyObject* t, int64_t units, int32_t& width) {
        int64_t s[2] = {};
        shape(t, s);
        width = narrow(s[1]);
        return ints(t, {units, s[1]});
    }
    void* rows(PyObject* t, PyObject* dtype, int64_t B, int64_t H, int64_t n, int64_t d, int64_t (&st)[3]) {     // [B, H, n, d], contiguous rows
        int64_t s[4] = {}, all[4] = {};
        shape(t, s);
        if (s[0] != B || s[1] != H || s[2] != n || s[3] != d) ok = false;
        typed(t, dtype);
        if (!ok) return nullptr;
        Ref r(method(t, s_stride));
        extents(r.p, all);
        if (all[3] != 1) ok = false;
        int64_t inner = d;                                   // an axis of one element has any stride in torch, and here that of a contiguous tensor
        for (int a = 2; a >= 0; --a) {
            st[a] = s[a] == 1 ? inner : all[a];
            inner *= s[a];
        }
        return placed(t);
    }
    zipvl_rope rope(PyObject* o) {                           // a ctypes structure
        zipvl_rope r = {};
        Py_buffer b;
        if (!ok || PyObject_GetBuffer(o, &b, PyBUF_SIMPLE)) { ok = false; return r; }
        if (b.len == (Py_ssize_t)sizeof r) memcpy(&r, b.buf, sizeof r);
        else ok = false;
        PyBuffer_Release(&b);
        return r;
    }
    struct Pool { zipvl_pages pages; int64_t d; PyObject* dtype; };
    Pool pool(PyObject* cache) {                             // a PagedCache
        Pool x = {};
        Ref K(PyObject_GetAttr(cache, s_K)), V(PyObject_GetAttr(cache, s_V));
        if (!K.p || !V.p) { ok = false; return x; }
        int64_t s[3] = {};
        shape(K.p, s);
        if (!ok) return x;
        Ref t(PyObject_GetAttr(K.p, s_dtype));
        if (t.p != g_f32 && t.p != g_bf16) { ok = false; return x; }
        x.dtype = t.p == g_f32 ? g_f32 : g_bf16;
        dense(K.p);
        x.pages.K = placed(K.p);
        x.pages.V = array(V.p, x.dtype, s);
        x.pages.num_pages = narrow(s[0]);
        x.pages.page = narrow(s[1]);
        x.d = s[2];
        return x;
    }
    void* stream_there() { return stream(true); }            // the current device's, if the tensors are on it
    void* stream(bool there = false) {                       // torch's current one
        if (!ok) return nullptr;
        Ref up(PyObject_CallNoArgs(g_is_initialized));
        if (up.p != Py_True) { ok = false; return nullptr; }
        Ref device(PyObject_CallNoArgs(g_get_device));
        if (!device.p || (there && PyLong_AsLong(device.p) != on)) { ok = false; return nullptr; }
        Ref s(PyObject_CallOneArg(g_get_stream, device.p));
        if (!s.p) { ok = false; return nullptr; }
        void* v = PyLong_AsVoidPtr(s.p);
        if (!v && PyErr_Occurred()) ok = false;
        return v;
    }
};

// What an argument raised the general way raises again; an interrupt (the calls into torch run Python code) would be lost.
PyObject* general_way() {
    if (PyErr_Occurred() && !PyErr_ExceptionMatches(PyExc_Exception)) return nullptr;
    PyErr_Clear();
    Py_RETURN_NONE;
}

// `call` runs without the GIL
template <typename F>
PyObject* finish(const Args& x, F&& call) {
    if (!x.ok) return general_way();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

bool count_is(Py_ssize_t n, Py_ssize_t want) { return n == want; }

// (Q, K, probe_pos, scale, flags, mass, rank, ws)
PyObject* score(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 8)) return general_way();
    Args x{a};
    const zipvl_dims d = x.layer(a[0], a[1], nullptr);
    int32_t probes[ZIPVL_MAX_PROBES];
    const bool list = PyList_CheckExact(a[2]), seq = list || PyTuple_CheckExact(a[2]);
    const Py_ssize_t m = seq ? PySequence_Fast_GET_SIZE(a[2]) : 0;
    if (m < 1 || m > ZIPVL_MAX_PROBES) return general_way();
    for (Py_ssize_t i = 0; i < m; ++i) probes[i] = x.int32(PySequence_Fast_GET_ITEM(a[2], i));
    const float scale = (float)x.real(a[3]);
    const int flags = x.int32(a[4]);
    x.dense(a[5]);
    x.dense(a[6]);
    void *q = x.address(a[0]), *k = x.address(a[1]), *mass = x.address(a[5]), *rank = x.address_or_null(a[6]), *ws = x.address(a[7]);
    const size_t ws_bytes = x.bytes(a[7]);
    void* st = x.stream();
    return finish(x, [&] { return zipvl_score(q, k, &d, probes, (int)m, scale, flags, (float*)mass, (float*)rank, ws, ws_bytes, st); });
}

// (mass, rank, tau, idx, k, status, ws)
PyObject* select(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 7)) return general_way();
    Args x{a};
    int64_t s[2] = {};
    x.shape(a[0], s);
    const int units = x.narrow(s[0]), n = x.narrow(s[1]);
    const double tau = x.real(a[2]);
    x.dense(a[0]);
    x.dense(a[1]);
    x.dense(a[3]);
    x.dense(a[4]);
    void *mass = x.address(a[0]), *rank = x.address_or_null(a[1]), *idx = x.address(a[3]), *k = x.address(a[4]);
    void *status = x.address_or_null(a[5]), *ws = x.address_or_null(a[6]);
    const size_t ws_bytes = a[6] == Py_None ? 0 : x.bytes(a[6]);
    void* st = x.stream();
    return finish(x, [&] { return zipvl_select((float*)mass, (float*)rank, units, n, tau, (int32_t*)idx, (int32_t*)k, (int32_t*)status, ws, ws_bytes, st); });
}

// (K, V, idx, k, cap, flags, Kc, Vc, len)
PyObject* compact_kv(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 9)) return general_way();
    Args x{a};
    const zipvl_dims d = x.layer(nullptr, a[0], a[1]);
    const int cap = x.int32(a[4]), flags = x.int32(a[5]);
    void *K = x.address(a[0]), *V = x.address(a[1]), *idx = x.address_or_null(a[2]), *k = x.address_or_null(a[3]);
    void *Kc = x.address(a[6]), *Vc = x.address(a[7]), *len = x.address(a[8]);
    void* st = x.stream();
    return finish(x, [&] { return zipvl_compact_kv(K, V, &d, (int32_t*)idx, (int32_t*)k, Kc, Vc, cap, (int32_t*)len, flags, st); });
}

// (Q, K, V, idx, k, scale, flags, O, ws)
PyObject* sparse_prefill(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 9)) return general_way();
    Args x{a};
    const zipvl_dims d = x.layer(a[0], a[1], a[2]);
    const float scale = (float)x.real(a[5]);
    const int flags = x.int32(a[6]);
    void *Q = x.address(a[0]), *K = x.address(a[1]), *V = x.address(a[2]), *idx = x.address_or_null(a[3]), *k = x.address_or_null(a[4]);
    void *O = x.address(a[7]), *ws = x.address(a[8]);
    const size_t ws_bytes = x.bytes(a[8]);
    void* st = x.stream();
    return finish(x, [&] { return zipvl_sparse_prefill(Q, K, V, &d, (int32_t*)idx, (int32_t*)k, scale, flags, O, ws, ws_bytes, st); });
}

// (Kc, Vc, len, k_new, v_new, B, Hkv)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 7)) return general_way();
    Args x{a};
    int64_t s[3] = {};
    x.shape(a[0], s);
    const zipvl_dims d = x.step(a[5], a[6], a[6], s[1], s[2], x.dtype(a[0]));
    void *Kc = x.address(a[0]), *Vc = x.address(a[1]), *len = x.address(a[2]), *kn = x.address(a[3]), *vn = x.address(a[4]);
    void* st = x.stream();
    return finish(x, [&] { return zipvl_kv_append(Kc, Vc, (int32_t*)len, d.n, kn, vn, &d, st); });
}

// (q, Kc, Vc, len, k_new, v_new, scale, B, Hq, Hkv, ws, o)
PyObject* decode_step(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 12)) return general_way();
    Args x{a};
    int64_t s[3] = {};
    x.shape(a[1], s);
    const zipvl_dims d = x.step(a[7], a[8], a[9], s[1], s[2], x.dtype(a[1]));
    const float scale = (float)x.real(a[6]);
    void *q = x.address(a[0]), *Kc = x.address(a[1]), *Vc = x.address(a[2]), *len = x.address(a[3]), *kn = x.address(a[4]), *vn = x.address(a[5]);
    void *ws = x.address(a[10]), *o = x.address(a[11]);
    const size_t ws_bytes = x.bytes(a[10]);
    void* st = x.stream();
    return finish(x, [&] { return zipvl_decode_step(q, Kc, Vc, (int32_t*)len, d.n, kn, vn, &d, scale, o, ws, ws_bytes, st); });
}

// (q, cache, scale, B, Hq, Hkv, K_tail, V_tail, len_tail, o, ws)
PyObject* decode_attn_q(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 11)) return general_way();
    Args x{a};
    Ref K(PyObject_GetAttr(a[1], s_K)), V(PyObject_GetAttr(a[1], s_V)), lh(PyObject_GetAttr(a[1], s_len_hi)), ll(PyObject_GetAttr(a[1], s_len_lo));
    Ref ch(PyObject_GetAttr(a[1], s_cap_hi)), cl(PyObject_GetAttr(a[1], s_cap_lo)), dd(PyObject_GetAttr(a[1], s_d));
    if (!K.p || !V.p || !lh.p || !ll.p || !ch.p || !cl.p || !dd.p || !PyDict_CheckExact(K.p) || !PyDict_CheckExact(V.p)) return general_way();
    auto parts = [&](PyObject* dict) {
        auto part = [&](PyObject* name) -> void* {
            if (!x.ok) return nullptr;
            PyObject* t = PyDict_GetItemWithError(dict, name);
            if (!t) { x.ok = false; return nullptr; }
            return x.address(t);
        };
        zipvl_qtensor t;
        t.hi_codes = decltype(t.hi_codes)(part(s_hi_codes));
        t.hi_params = decltype(t.hi_params)(part(s_hi_params));
        t.lo_codes = decltype(t.lo_codes)(part(s_lo_codes));
        t.lo_params = decltype(t.lo_params)(part(s_lo_params));
        return t;
    };
    const zipvl_qtensor kq = parts(K.p), vq = parts(V.p);
    const int cap_hi = x.int32(ch.p), cap_lo = x.int32(cl.p);
    int64_t s[3] = {};
    if (a[6] != Py_None) x.shape(a[6], s);
    const zipvl_dims d = x.step(a[3], a[4], a[5], (int64_t)cap_hi + cap_lo + s[1], x.number(dd.p), x.dtype(a[0]));
    const float scale = (float)x.real(a[2]);
    void *q = x.address(a[0]), *hi = x.address(lh.p), *lo = x.address(ll.p), *Kt = x.address_or_null(a[6]), *Vt = x.address_or_null(a[7]);
    void *lt = x.address_or_null(a[8]), *o = x.address(a[9]), *ws = x.address(a[10]);
    const size_t ws_bytes = x.bytes(a[10]);
    const int cap_tail = x.narrow(s[1]);
    void* st = x.stream();
    return finish(x, [&] {
        return zipvl_decode_attn_q(q, &kq, &vq, (int32_t*)hi, (int32_t*)lo, cap_hi, cap_lo, Kt, Vt, (int32_t*)lt, cap_tail, &d, scale, o, ws, ws_bytes, st);
    });
}

// (Q, K, pos, rope, flags, Qo, Ko); Q with Qo or K with Ko may be None
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 7)) return general_way();
    Args x{a};
    const bool q = a[0] != Py_None, k = a[1] != Py_None;
    if ((!q && !k) || q != (a[5] != Py_None) || k != (a[6] != Py_None)) return general_way();
    zipvl_dims d = {}, out = {};
    int64_t s[4] = {}, sk[4] = {};
    x.shape(a[q ? 0 : 1], s);
    if (k) x.shape(a[1], sk);
    d.B = x.narrow(s[0]); d.n = x.narrow(s[2]); d.d = x.narrow(s[3]);
    d.Hkv = x.narrow(k ? sk[1] : s[1]);
    d.Hq = x.narrow(s[1]);
    d.dtype = x.dtype(a[q ? 0 : 1]);
    PyObject* type = d.dtype ? g_bf16 : g_f32;
    out = d;
    void *Q = q ? x.rows(a[0], type, s[0], s[1], s[2], s[3], d.q_strides) : nullptr, *Qo = q ? x.rows(a[5], type, s[0], s[1], s[2], s[3], out.q_strides) : nullptr;
    void *K = k ? x.rows(a[1], type, s[0], sk[1], s[2], s[3], d.k_strides) : nullptr, *Ko = k ? x.rows(a[6], type, s[0], sk[1], s[2], s[3], out.k_strides) : nullptr;
    const zipvl_rope rope = x.rope(a[3]);
    void* pos = x.ints(a[2], {(int64_t)rope.axes, s[0], s[2]});
    const int flags = x.int32(a[4]);
    void* st = x.stream_there();
    return finish(x, [&] { return zipvl_rotate(Q, K, &d, (int32_t*)pos, &rope, flags, Qo, Ko, &out, st); });
}

// (K, V, cache, table, start, idx, k, pos, rope, Q, Qo, length, flags)
PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 13)) return general_way();
    Args x{a};
    const bool q = a[9] != Py_None, turned = a[8] != Py_None;
    if (q != (a[10] != Py_None)) return general_way();
    zipvl_dims d = {};
    int64_t s[4] = {}, sq[4] = {};
    x.shape(a[0], s);
    if (q) x.shape(a[9], sq);
    d.B = x.narrow(s[0]); d.Hkv = x.narrow(s[1]); d.n = x.narrow(s[2]); d.d = x.narrow(s[3]);
    d.Hq = q ? x.narrow(sq[1]) : d.Hkv;
    d.dtype = x.dtype(a[0]);
    PyObject* type = d.dtype ? g_bf16 : g_f32;
    const Args::Pool pool = x.pool(a[2]);
    if (pool.dtype != type || pool.d != s[3]) return general_way();
    void *K = x.rows(a[0], type, s[0], s[1], s[2], s[3], d.k_strides), *V = x.rows(a[1], type, s[0], s[1], s[2], s[3], d.v_strides);
    const int flags = x.int32(a[12]);
    const int64_t units = s[0] * s[1], sets = flags & ZIPVL_T_PER_BATCH ? s[0] : units;
    int32_t width = 0;
    void *table = x.table(a[3], units, width), *start = x.ints(a[4], {units}), *len = a[11] == a[4] ? start : x.ints(a[11], {units});
    void *idx = x.ints_or_null(a[5], {sets, s[2]}), *k = x.ints_or_null(a[6], {sets});
    zipvl_rope rope = {};
    if (turned) rope = x.rope(a[8]);
    void* pos = turned ? x.ints(a[7], {(int64_t)rope.axes, s[0], s[2]}) : nullptr;
    void *Q = nullptr, *Qo = nullptr;
    if (q) {
        Q = x.rows(a[9], type, s[0], sq[1], s[2], s[3], d.q_strides);
        Qo = x.array(a[10], type, {s[0], sq[1], s[2], s[3]});
    }
    void* st = x.stream_there();
    return finish(x, [&] {
        return zipvl_paged_append(K, V, &d, (int32_t*)idx, (int32_t*)k, (int32_t*)pos, turned ? &rope : nullptr, &pool.pages, (int32_t*)table, width,
                                  (int32_t*)start, (int32_t*)len, Q, Qo, flags, st);
    });
}

// (q, cache, table, length, scale, B, Hq, Hkv, prefix_table, prefix_len, group_begin, o, ws)
PyObject* decode_attn_paged(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 13)) return general_way();
    Args x{a};
    const Args::Pool pool = x.pool(a[1]);
    const zipvl_dims d = x.step(a[5], a[6], a[7], 1, pool.d, pool.dtype == g_bf16);
    const float scale = (float)x.real(a[4]);
    auto heads = [&](PyObject* t) {                          // any contiguous shape of B Hq rows
        if ((int64_t)x.bytes(t) != (int64_t)d.B * d.Hq * d.d) x.ok = false;
        x.typed(t, pool.dtype);
        x.dense(t);
        return x.placed(t);
    };
    void *q = heads(a[0]), *o = heads(a[11]);
    const int64_t units = (int64_t)d.B * d.Hkv;
    int32_t width = 0, prefix_width = 0, groups = 0;
    void *table = x.table(a[2], units, width), *len = x.ints(a[3], {units}), *prefix_table = nullptr, *prefix_len = nullptr, *begin = nullptr;
    if (a[8] != Py_None || a[9] != Py_None || a[10] != Py_None) {
        int64_t s[1] = {};
        x.shape(a[10], s);
        groups = x.narrow(s[0] - 1);
        if (groups < 1) x.ok = false;
        prefix_table = x.table(a[8], (int64_t)groups * d.Hkv, prefix_width);
        prefix_len = x.ints(a[9], {(int64_t)groups * d.Hkv});
        begin = x.ints(a[10], {(int64_t)groups + 1});
    }
    x.typed(a[12], g_u8);
    x.dense(a[12]);
    void* ws = x.placed(a[12]);
    const size_t ws_bytes = x.bytes(a[12]);
    void* st = x.stream_there();
    return finish(x, [&] {
        return zipvl_decode_attn_paged(q, &pool.pages, (int32_t*)table, width, (int32_t*)len, (int32_t*)prefix_table, prefix_width, (int32_t*)prefix_len,
                                       (int32_t*)begin, groups, &d, scale, o, ws, ws_bytes, st);
    });
}

// Queries [B, H, n, d] against the units of a table: dims with Q's strides, and what stands beside it.
struct Queries { zipvl_dims d; void *Q, *table, *len, *k; int32_t width; int64_t units, s[4]; PyObject* type; };
Queries queries(Args& x, const Args::Pool& pool, PyObject* Q, PyObject* table, PyObject* length, PyObject* k) {
    Queries q = {};
    x.shape(Q, q.s);
    q.type = pool.dtype;
    if (!x.ok || q.s[3] != pool.d || q.s[0] < 1) { x.ok = false; return q; }
    int64_t t[2] = {};
    x.shape(table, t);
    q.units = t[0];
    if (q.units < 1 || q.units % q.s[0]) x.ok = false;
    q.d.B = x.narrow(q.s[0]); q.d.Hq = x.narrow(q.s[1]); q.d.n = x.narrow(q.s[2]); q.d.d = x.narrow(q.s[3]);
    q.d.Hkv = x.ok ? x.narrow(q.units / q.s[0]) : 0;
    q.d.dtype = q.type == g_bf16;
    q.Q = x.rows(Q, q.type, q.s[0], q.s[1], q.s[2], q.s[3], q.d.q_strides);
    q.table = x.table(table, q.units, q.width);
    q.len = x.ints(length, {q.units});
    q.k = x.ints_or_null(k, {q.units});
    return q;
}

// (Q, cache, table, length, scale, k, prefix_table, prefix_len, group_begin, O, lse, ws)
PyObject* chunk_attn_paged(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 12)) return general_way();
    Args x{a};
    const Args::Pool pool = x.pool(a[1]);
    if (!x.ok) return general_way();
    Queries q = queries(x, pool, a[0], a[2], a[3], a[5]);
    const float scale = (float)x.real(a[4]);
    int32_t prefix_width = 0, groups = 0;
    void *prefix_table = nullptr, *prefix_len = nullptr, *begin = nullptr;
    if (a[6] != Py_None || a[7] != Py_None || a[8] != Py_None) {
        int64_t s[1] = {};
        x.shape(a[8], s);
        groups = x.narrow(s[0] - 1);
        if (groups < 1) x.ok = false;
        prefix_table = x.table(a[6], (int64_t)groups * q.d.Hkv, prefix_width);
        prefix_len = x.ints(a[7], {(int64_t)groups * q.d.Hkv});
        begin = x.ints(a[8], {(int64_t)groups + 1});
    }
    zipvl_dims out = q.d;
    void* O = x.rows(a[9], q.type, q.s[0], q.s[1], q.s[2], q.s[3], out.q_strides);
    void* lse = a[10] == Py_None ? nullptr : x.array(a[10], g_f32, {q.s[0], q.s[1], q.s[2]});
    x.typed(a[11], g_u8);
    x.dense(a[11]);
    void* ws = x.placed(a[11]);
    const size_t ws_bytes = x.bytes(a[11]);
    void* st = x.stream_there();
    return finish(x, [&] {
        return zipvl_chunk_attn_paged(q.Q, &pool.pages, (int32_t*)q.table, q.width, (int32_t*)q.len, (int32_t*)q.k, (int32_t*)prefix_table, prefix_width, (int32_t*)prefix_len,
                                      (int32_t*)begin, groups, &q.d, scale, O, &out, (float*)lse, ws, ws_bytes, st);
    });
}

// (Q, cache, table, length, lse, scale, k, before, weight)
PyObject* paged_weigh(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 9)) return general_way();
    Args x{a};
    const Args::Pool pool = x.pool(a[1]);
    if (!x.ok) return general_way();
    Queries q = queries(x, pool, a[0], a[2], a[3], a[6]);
    const float scale = (float)x.real(a[5]);
    void* lse = x.array(a[4], g_f32, {q.s[0], q.s[1], q.s[2]});          // a view of some of the tokens goes the general way
    const int64_t room = (int64_t)q.width * pool.pages.page;
    void* weight = x.array(a[8], g_f32, {q.units, room});
    void* before = a[7] == Py_None ? nullptr : a[7] == a[8] ? weight : x.array(a[7], g_f32, {q.units, room});
    void* st = x.stream_there();
    return finish(x, [&] {
        return zipvl_paged_weigh(q.Q, &pool.pages, (int32_t*)q.table, q.width, (int32_t*)q.len, (int32_t*)q.k, (float*)lse, q.s[2], &q.d, scale, (float*)before,
                                 (float*)weight, st);
    });
}

// (cache, table, length, k, weight, tokens, budget, sinks, recent, length_out, weight_out, tokens_out, ws)
PyObject* paged_evict(PyObject*, PyObject* const* a, Py_ssize_t na) {
    if (!count_is(na, 13)) return general_way();
    Args x{a};
    const Args::Pool pool = x.pool(a[0]);
    int64_t t[2] = {};
    x.shape(a[1], t);
    if (!x.ok) return general_way();
    const int64_t units = t[0], room = t[1] * pool.pages.page;
    zipvl_dims d = {};
    d.B = x.narrow(units); d.Hq = d.Hkv = d.n = 1; d.d = x.narrow(pool.d);
    d.dtype = pool.dtype == g_bf16;
    int32_t width = 0;
    void *table = x.table(a[1], units, width), *len = x.ints(a[2], {units}), *k = x.ints_or_null(a[3], {units});
    void *weight = x.array(a[4], g_f32, {units, room}), *tokens = x.ints_or_null(a[5], {units, room});
    const int budget = x.int32(a[6]), sinks = x.int32(a[7]), recent = x.int32(a[8]);
    void* len_out = a[9] == a[2] ? len : x.ints(a[9], {units});
    void* weight_out = a[10] == a[4] ? weight : x.array(a[10], g_f32, {units, room});
    void* tokens_out = a[11] == a[5] ? tokens : x.ints_or_null(a[11], {units, room});
    x.typed(a[12], g_u8);
    x.dense(a[12]);
    void* ws = x.placed(a[12]);
    const size_t ws_bytes = x.bytes(a[12]);
    void* st = x.stream_there();
    return finish(x, [&] {
        return zipvl_paged_evict(&pool.pages, (int32_t*)table, width, &d, (int32_t*)len, (int32_t*)k, (float*)weight, (int32_t*)tokens, budget, sinks, recent,
                                 (int32_t*)len_out, (float*)weight_out, (int32_t*)tokens_out, ws, ws_bytes, st);
    });
}

#define ZIPVL_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ZIPVL_METHOD(score), ZIPVL_METHOD(select), ZIPVL_METHOD(compact_kv), ZIPVL_METHOD(sparse_prefill), ZIPVL_METHOD(kv_append),
                         ZIPVL_METHOD(decode_step), ZIPVL_METHOD(decode_attn_q), ZIPVL_METHOD(rotate), ZIPVL_METHOD(paged_append),
                         ZIPVL_METHOD(decode_attn_paged), ZIPVL_METHOD(chunk_attn_paged), ZIPVL_METHOD(paged_weigh), ZIPVL_METHOD(paged_evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pycall", "Calls of libzipvl.so on torch tensors", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pycall(void) {
    struct { PyObject** at; const char* text; } names[] = {
        {&s_data_ptr, "data_ptr"}, {&s_shape, "shape"}, {&s_dtype, "dtype"}, {&s_stride, "stride"}, {&s_numel, "numel"}, {&s_is_contiguous, "is_contiguous"},
        {&s_hi_codes, "hi_codes"}, {&s_hi_params, "hi_params"}, {&s_lo_codes, "lo_codes"}, {&s_lo_params, "lo_params"}, {&s_K, "K"}, {&s_V, "V"},
        {&s_len_hi, "len_hi"}, {&s_len_lo, "len_lo"}, {&s_cap_hi, "cap_hi"}, {&s_cap_lo, "cap_lo"}, {&s_d, "d"}, {&s_on_device, "get_device"}};
    for (auto& n : names)
        if (!(*n.at = PyUnicode_InternFromString(n.text))) return nullptr;
    Ref torch(PyImport_ImportModule("torch"));
    if (!torch.p) return nullptr;
    struct { PyObject** at; const char *in, *name; } objects[] = {
        {&g_tensor, nullptr, "Tensor"}, {&g_f32, nullptr, "float32"}, {&g_bf16, nullptr, "bfloat16"}, {&g_i32, nullptr, "int32"}, {&g_u8, nullptr, "uint8"}, {&g_is_initialized, "cuda", "is_initialized"},
        {&g_get_device, "_C", "_cuda_getDevice"}, {&g_get_stream, "_C", "_cuda_getCurrentRawStream"}};
    for (auto& o : objects) {
        Ref in(o.in ? PyObject_GetAttrString(torch.p, o.in) : nullptr);
        if (o.in && !in.p) return nullptr;
        if (!(*o.at = PyObject_GetAttrString(o.in ? in.p : torch.p, o.name))) return nullptr;
    }
    return PyModule_Create(&module);
}

// marshal.cpp -- the short way from torch tensors to the C entry points, for the ordinary call.
//
// A call of the binding spends 9 us in Python besides the 3.6 us of the C entry point itself (attribute look-ups,
// two allocations, the current stream, ctypes conversions), which is more than the kernels of a small call take.  The
// functions here do the same for a call whose arguments are plain contiguous tensors on one GPU, and return None for
// every other one without having done anything: the binding's Python code then handles it, errors included.  Host
// only; the entry points' addresses come from the binding (set_entries), so nothing links to the library.
#include <ATen/ATen.h>
#include <Python.h>
#include <c10/core/DeviceGuard.h>
#include <pybind11/gil.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cmath>

namespace {

typedef int (*FwdFn)(const void *, const void *, const void *, void *, float *, int, int, int, int, int, int, float, void *);
typedef int (*SplitFn)(const void *, const void *, const void *, void *, float *, void *, long long, int, int, int, int, int,
                       int, int, float, void *);
typedef int (*BwdFn)(const void *, const void *, const void *, const void *, const void *, const float *, void *, void *,
                     void *, float *, int, int, int, int, int, int, float, void *);
typedef long long (*WsFn)(int, int, int, int, int);

// [0] bf16, [1] fp16
FwdFn g_fwd[2];
SplitFn g_split[2];
BwdFn g_bwd[2];
WsFn g_ws;
PyObject *g_current_stream;   // device index -> address of its current stream

const at::ScalarType kElem[2] = {at::kBFloat16, at::kHalf};

// a plain contiguous GPU tensor of this type (no subclass, nothing without memory of its own)
const at::Tensor *plain(PyObject *o, at::ScalarType type, int64_t dims)
{
    if (!THPVariable_CheckExact(o))
        return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.scalar_type() != type ||
        (dims && t.dim() != dims) || !t.is_contiguous() || t.is_conj() || t.is_neg())
        return nullptr;
    return &t;
}

struct Shape {
    int B, H, S_q, S_kv, D;
};

bool same_shape(const at::Tensor &a, const at::Tensor &b) { return a.sizes() == b.sizes() && a.device() == b.device(); }

// q [B,H,S_q,D], k and v [B,H,S_kv,D] on one device, sizes the entry points can count
bool qkv(PyObject *const *a, at::ScalarType type, const at::Tensor *t[3], Shape &s)
{
    for (int i = 0; i < 3; ++i)
        if (!(t[i] = plain(a[i], type, 4)))
            return false;
    const auto q = t[0]->sizes(), k = t[1]->sizes();
    if (!same_shape(*t[1], *t[2]) || t[0]->device() != t[1]->device() || k[0] != q[0] || k[1] != q[1] || k[3] != q[3])
        return false;
    for (int i = 0; i < 4; ++i)
        if (q[i] < 1 || k[i] < 1 || q[i] > INT_MAX || k[i] > INT_MAX)
            return false;
    s = {(int)q[0], (int)q[1], (int)q[2], (int)k[2], (int)q[3]};
    return true;
}

bool is_lse(const at::Tensor &t, const Shape &s, const at::Tensor &q)
{
    return t.size(0) == s.B && t.size(1) == s.H && t.size(2) == s.S_q && t.device() == q.device();
}

bool scale_of(PyObject *o, int D, float &scale)
{
    if (o == Py_None)
        scale = (float)(1.0 / std::pow((double)D, 0.5));
    else if (PyFloat_CheckExact(o))
        scale = (float)PyFloat_AS_DOUBLE(o);
    else
        return false;
    return true;
}

// the address in a Python int (the reference is taken over)
bool address_of(PyObject *h, void *&address)
{
    address = h && PyLong_CheckExact(h) ? PyLong_AsVoidPtr(h) : nullptr;
    const bool ok = h && PyLong_CheckExact(h) && !PyErr_Occurred();
    Py_XDECREF(h);
    PyErr_Clear();
    return ok;
}

// The stream to launch on: the device's current one, or the one the caller names.  `allocates`: the call has something to
// allocate, and what is allocated here belongs to the current stream; a call that needs memory of another stream goes the
// other way.
bool stream_of(PyObject *o, const c10::Device &dev, bool allocates, void *&stream)
{
    void *current = nullptr;
    if (o == Py_None || allocates) {
        PyObject *index = PyLong_FromLong(dev.index());
        const bool ok = address_of(index && g_current_stream ? PyObject_CallOneArg(g_current_stream, index) : nullptr, current);
        Py_XDECREF(index);
        if (!ok)
            return false;
        if (o == Py_None) {
            stream = current;
            return true;
        }
    }
    return address_of(PyObject_GetAttrString(o, "cuda_stream"), stream) && (!allocates || stream == current);
}

// one of these arguments is left for the call to allocate
bool any_none(PyObject *const *a, int n)
{
    for (int i = 0; i < n; ++i)
        if (a[i] == Py_None)
            return true;
    return false;
}

// the launch, with the tensors' device current and the interpreter lock released
template <typename F>
int launch(const c10::Device &dev, F f)
{
    const c10::OptionalDeviceGuard guard(dev);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

PyObject *pack(std::initializer_list<const at::Tensor *> ts)
{
    PyObject *r = PyTuple_New((Py_ssize_t)ts.size());
    Py_ssize_t i = 0;
    for (const at::Tensor *t : ts) {
        PyObject *w = r ? THPVariable_Wrap(*t) : nullptr;
        if (!w) {
            Py_XDECREF(r);
            return nullptr;
        }
        PyTuple_SET_ITEM(r, i++, w);
    }
    return r;
}

// An allocation, with the interpreter lock released as torch's own functions do it: it may wait for the device, and other
// threads of the program (host callbacks of queued work among them) must be able to run meanwhile.
template <typename F>
at::Tensor allocate(F make)
{
    const pybind11::gil_scoped_release no_gil;
    return make();
}

// an output the caller may have given: taken as it is, or allocated like `like`; false if it needs the other way
bool output(PyObject *given, const at::Tensor &like, at::Tensor &out)
{
    if (given == Py_None) {
        out = allocate([&] { return at::empty_like(like); });
        return true;
    }
    const at::Tensor *t = plain(given, like.scalar_type(), 0);
    if (!t || !same_shape(*t, like))
        return false;
    out = *t;
    return true;
}

bool lse_output(PyObject *given, const Shape &s, const at::Tensor &q, at::Tensor &out)
{
    if (given == Py_None) {
        out = allocate([&] { return at::empty({s.B, s.H, s.S_q}, q.options().dtype(at::kFloat)); });
        return true;
    }
    const at::Tensor *t = plain(given, at::kFloat, 3);
    if (!t || !is_lse(*t, s, q))
        return false;
    out = *t;
    return true;
}

// True / False, or a truth value another object would have to be asked for
int truth(PyObject *o) { return o == Py_True ? 1 : o == Py_False ? 0 : -1; }

// 0 for bf16, 1 for fp16
int type_of(PyObject *o) { return (int)PyLong_AsLong(o) & 1; }

// fwd(type, q, k, v, o, lse, causal, scale, stream) -> (o, lse), a status other than 0, or None
PyObject *py_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *t[3];
    Shape s;
    float scale;
    void *stream;
    at::Tensor o, lse;
    const int type = n == 9 ? type_of(a[0]) : 0, causal = n == 9 ? truth(a[6]) : -1;
    if (n != 9 || causal < 0 || !g_fwd[type] || !qkv(a + 1, kElem[type], t, s) || !scale_of(a[7], s.D, scale) ||
        !stream_of(a[8], t[0]->device(), any_none(a + 4, 2), stream) || !output(a[4], *t[0], o) || !lse_output(a[5], s, *t[0], lse))
        Py_RETURN_NONE;
    const int rc = launch(t[0]->device(), [&] {
        return g_fwd[type](t[0]->data_ptr(), t[1]->data_ptr(), t[2]->data_ptr(), o.data_ptr(), (float *)lse.data_ptr(), s.B,
                           s.H, s.S_q, s.S_kv, s.D, causal, scale, stream);
    });
    return rc ? PyLong_FromLong(rc) : pack({&o, &lse});
    END_HANDLE_TH_ERRORS
}

// splitkv(type, q, k, v, n_split, o, lse, workspace, causal, scale, stream)
PyObject *py_splitkv(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *t[3];
    Shape s;
    float scale;
    void *stream;
    at::Tensor o, lse, ws;
    const int type = n == 11 ? type_of(a[0]) : 0, causal = n == 11 ? truth(a[8]) : -1;
    if (n != 11 || causal < 0 || !g_split[type] || !g_ws || !PyLong_CheckExact(a[4]) || !qkv(a + 1, kElem[type], t, s) ||
        !scale_of(a[9], s.D, scale) || !stream_of(a[10], t[0]->device(), any_none(a + 5, 3), stream))
        Py_RETURN_NONE;
    const long n_split = PyLong_AsLong(a[4]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const long long need = n_split >= 1 && n_split <= 256 ? g_ws(s.B, s.H, s.S_q, s.D, (int)n_split) : -1;
    if (need < 1)
        Py_RETURN_NONE;
    if (a[7] != Py_None) {
        if (!THPVariable_CheckExact(a[7]))
            Py_RETURN_NONE;
        ws = THPVariable_Unpack(a[7]);
        if (!plain(a[7], ws.scalar_type(), 0) || ws.device() != t[0]->device())
            Py_RETURN_NONE;
    }
    if (!output(a[5], *t[0], o) || !lse_output(a[6], s, *t[0], lse))
        Py_RETURN_NONE;
    if (!ws.defined())
        ws = allocate([&] { return at::empty({need < 16 ? 16 : need}, t[0]->options().dtype(at::kByte)); });
    const int rc = launch(t[0]->device(), [&] {
        return g_split[type](t[0]->data_ptr(), t[1]->data_ptr(), t[2]->data_ptr(), o.data_ptr(), (float *)lse.data_ptr(),
                             ws.data_ptr(), (long long)ws.nbytes(), (int)n_split, s.B, s.H, s.S_q, s.S_kv, s.D, causal, scale,
                             stream);
    });
    return rc ? PyLong_FromLong(rc) : pack({&o, &lse});
    END_HANDLE_TH_ERRORS
}

// bwd(type, q, k, v, o, d_o, lse, dq, dk, dv, delta_ws, causal, scale, stream)
PyObject *py_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const at::Tensor *t[3];
    Shape s;
    float scale;
    void *stream;
    at::Tensor g[3], ws;
    const int type = n == 14 ? type_of(a[0]) : 0, causal = n == 14 ? truth(a[11]) : -1;
    if (n != 14 || causal < 0 || !g_bwd[type] || !qkv(a + 1, kElem[type], t, s) || !scale_of(a[12], s.D, scale) ||
        !stream_of(a[13], t[0]->device(), any_none(a + 7, 4), stream))
        Py_RETURN_NONE;
    const at::Tensor *o = plain(a[4], kElem[type], 4), *d_o = plain(a[5], kElem[type], 4), *lse = plain(a[6], at::kFloat, 3);
    if (!o || !d_o || !lse || !same_shape(*o, *t[0]) || !same_shape(*d_o, *t[0]) || !is_lse(*lse, s, *t[0]))
        Py_RETURN_NONE;
    const int64_t rows2 = 2ll * s.B * s.H * s.S_q;
    if (a[10] != Py_None) {
        const at::Tensor *w = plain(a[10], at::kFloat, 0);
        if (!w || w->numel() < rows2 || w->device() != t[0]->device())
            Py_RETURN_NONE;
        ws = *w;
    }
    for (int i = 0; i < 3; ++i)
        if (!output(a[7 + i], *t[i], g[i]))
            Py_RETURN_NONE;
    if (!ws.defined())
        ws = allocate([&] { return at::empty({rows2}, t[0]->options().dtype(at::kFloat)); });
    const int rc = launch(t[0]->device(), [&] {
        return g_bwd[type](t[0]->data_ptr(), t[1]->data_ptr(), t[2]->data_ptr(), o->data_ptr(), d_o->data_ptr(),
                           (const float *)lse->data_ptr(), g[0].data_ptr(), g[1].data_ptr(), g[2].data_ptr(),
                           (float *)ws.data_ptr(), s.B, s.H, s.S_q, s.S_kv, s.D, causal, scale, stream);
    });
    return rc ? PyLong_FromLong(rc) : pack({&g[0], &g[1], &g[2]});
    END_HANDLE_TH_ERRORS
}

// ---- rotary positions, the paged cache and attention over it

typedef int (*RopeFn)(const void *, void *, const void *, void *, const long long *, const int *, const double *, const int *, int,
                      int, int, int, int, int, int, int, void *);
typedef int (*WriteFn)(const void *, const void *, const long long *, void *, void *, unsigned char *, unsigned char *,
                       const int *, const int *, const int *, int, int, int, int, int, int, int, int, void *);
typedef int (*ReadFn)(void *, void *, const long long *, const void *, const void *, const unsigned char *,
                      const unsigned char *, const int *, const int *, const int *, int, int, int, int, int, int, int, int, void *);
typedef int (*PagedFn)(const void *, const long long *, void *, float *, const void *, const void *, const unsigned char *,
                       const unsigned char *, const int *, const int *, const int *, int, void *, long long, int, int, int, int,
                       int, int, int, int, int, int, float, void *);
typedef long long (*PagedWsFn)(int, int, int, int, int);

RopeFn g_rope[2];
WriteFn g_write[2];
ReadFn g_read[2];
PagedFn g_paged[2];
PagedWsFn g_paged_ws;

// a GPU tensor of rows of contiguous elements, any strides between the rows
const at::Tensor *rows_of(PyObject *o, at::ScalarType type, int64_t dims)
{
    if (!THPVariable_CheckExact(o))
        return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() || t.scalar_type() != type ||
        t.dim() != dims || t.is_conj() || t.is_neg())
        return nullptr;
    for (int64_t d = 0; d < dims; ++d)
        if (t.size(d) < 1 || t.size(d) > INT_MAX)
            return nullptr;
    return t.size(dims - 1) == 1 || t.stride(dims - 1) == 1 ? &t : nullptr;
}

// no two rows of it share memory: sorted by stride, every dimension steps over the ones below it
bool disjoint(const at::Tensor &t)
{
    int64_t dims[8][2], n = 0, reach = 1;
    if (t.dim() > 8)
        return false;
    for (int64_t d = 0; d < t.dim(); ++d) {
        if (t.size(d) < 2)
            continue;
        int64_t i = n++;
        for (; i > 0 && dims[i - 1][0] > t.stride(d); --i)
            dims[i][0] = dims[i - 1][0], dims[i][1] = dims[i - 1][1];
        dims[i][0] = t.stride(d), dims[i][1] = t.size(d);
    }
    for (int64_t i = 0; i < n; ++i) {
        if (dims[i][0] < reach)
            return false;
        reach += dims[i][0] * (dims[i][1] - 1);
    }
    return true;
}

long long stride_of(const at::Tensor &t, int64_t d) { return t.size(d) > 1 ? t.stride(d) : 0; }

// an output of rows that the caller may have given: as it is, or allocated contiguous in this shape
bool rows_output(PyObject *given, const at::Tensor &like, at::IntArrayRef shape, at::ScalarType type, at::Tensor &out)
{
    if (given == Py_None) {
        out = allocate([&] { return at::empty(shape, like.options().dtype(type)); });
        return true;
    }
    const at::Tensor *t = rows_of(given, type, (int64_t)shape.size());
    if (!t || t->sizes() != shape || t->device() != like.device() || !disjoint(*t))
        return false;
    out = *t;
    return true;
}

// whole numbers that a C int holds; false: the binding has to look at them
bool int_of(PyObject *o, int &x)
{
    if (!PyLong_CheckExact(o))
        return false;
    int overflow;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || v < INT_MIN || v > INT_MAX)
        return false;
    x = (int)v;
    return true;
}

// rope(type, q, k, pos, freq, sections, q_out, k_out, interleaved, inverse, stream) -> (q_out, k_out), a status or None
PyObject *py_rope(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const int type = n == 11 ? type_of(a[0]) : 0, inter = n == 11 ? truth(a[8]) : -1, inverse = n == 11 ? truth(a[9]) : -1;
    if (n != 11 || inter < 0 || inverse < 0 || !g_rope[type] || a[2] == Py_None ||
        (!PyList_CheckExact(a[5]) && !PyTuple_CheckExact(a[5])))
        Py_RETURN_NONE;
    const at::Tensor *q = rows_of(a[1], kElem[type], 4), *k = rows_of(a[2], kElem[type], 4);
    const at::Tensor *pos = plain(a[3], at::kInt, 3), *freq = plain(a[4], at::kDouble, 1);
    if (!q || !k || !pos || !freq || q->device() != k->device() || pos->device() != q->device() || freq->device() != q->device() ||
        k->size(0) != q->size(0) || k->size(2) != q->size(2) || k->size(3) != q->size(3))
        Py_RETURN_NONE;
    int sections[4];
    const Py_ssize_t axes = PySequence_Fast_GET_SIZE(a[5]);
    int64_t pairs = 0;
    if (axes < 1 || axes > 4)
        Py_RETURN_NONE;
    for (Py_ssize_t i = 0; i < axes; ++i) {
        if (!int_of(PySequence_Fast_GET_ITEM(a[5], i), sections[i]))
            Py_RETURN_NONE;
        pairs += sections[i];
    }
    void *stream;
    if (pos->size(0) != axes || pos->size(1) != q->size(0) || pos->size(2) != q->size(2) || freq->size(0) != pairs ||
        !stream_of(a[10], q->device(), any_none(a + 6, 2), stream))
        Py_RETURN_NONE;
    at::Tensor out[2];
    if (!rows_output(a[6], *q, q->sizes(), kElem[type], out[0]) || !rows_output(a[7], *k, k->sizes(), kElem[type], out[1]))
        Py_RETURN_NONE;
    long long strides[12];
    const at::Tensor *const four[4] = {q, &out[0], k, &out[1]};
    for (int i = 0; i < 12; ++i)
        strides[i] = stride_of(*four[i / 3], i % 3);
    const int rc = launch(q->device(), [&] {
        return g_rope[type](q->data_ptr(), out[0].data_ptr(), k->data_ptr(), out[1].data_ptr(), strides,
                            (const int *)pos->data_ptr(), (const double *)freq->data_ptr(), sections, (int)axes, (int)q->size(0),
                            (int)q->size(1), (int)k->size(1), (int)q->size(2), (int)q->size(3), inter, inverse, stream);
    });
    return rc ? PyLong_FromLong(rc) : pack({&out[0], &out[1]});
    END_HANDLE_TH_ERRORS
}

struct Cache {
    const at::Tensor *k, *v, *table, *start, *kv_len;
    unsigned char *k_scale, *v_scale;
    int kind, n_pages, H_kv, page, D, B, width;
};

// a[0..4] = k_pages, v_pages, page_table, start, kv_len, with the two scales
bool cache_of(PyObject *const *a, PyObject *k_scale, PyObject *v_scale, at::ScalarType type, Cache &c)
{
    const bool e4m3 = k_scale != Py_None;
    if (e4m3 != (v_scale != Py_None))
        return false;
    const at::ScalarType elem = e4m3 ? at::kFloat8_e4m3fn : type;
    c.k = plain(a[0], elem, 4), c.v = plain(a[1], elem, 4);
    c.table = plain(a[2], at::kInt, 2), c.start = plain(a[3], at::kInt, 1), c.kv_len = plain(a[4], at::kInt, 1);
    if (!c.k || !c.v || !c.table || !c.start || !c.kv_len || !same_shape(*c.k, *c.v))
        return false;
    const auto s = c.k->sizes(), t = c.table->sizes();
    for (int i = 0; i < 4; ++i)
        if (s[i] < 1 || s[i] > INT_MAX)
            return false;
    if (t[0] < 1 || t[0] >= INT_MAX || t[1] < 1 || t[1] > INT_MAX || c.start->size(0) != t[0] + 1 || c.kv_len->size(0) != t[0] ||
        c.table->device() != c.k->device() || c.start->device() != c.k->device() || c.kv_len->device() != c.k->device())
        return false;
    c.k_scale = c.v_scale = nullptr;
    if (e4m3)
        for (int i = 0; i < 2; ++i) {
            const at::Tensor *x = plain(i ? v_scale : k_scale, at::kByte, 3);
            if (!x || x->sizes() != s.slice(0, 3) || x->device() != c.k->device())
                return false;
            (i ? c.v_scale : c.k_scale) = (unsigned char *)x->data_ptr();
        }
    c.kind = e4m3;
    c.n_pages = (int)s[0], c.H_kv = (int)s[1], c.page = (int)s[2], c.D = (int)s[3], c.B = (int)t[0], c.width = (int)t[1];
    return true;
}

// write(type, k, v, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale, stream) -> (k_pages, v_pages)
PyObject *py_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const int type = n == 11 ? type_of(a[0]) : 0;
    Cache c;
    void *stream;
    if (n != 11 || !g_write[type] || !cache_of(a + 3, a[8], a[9], kElem[type], c))
        Py_RETURN_NONE;
    const at::Tensor *k = rows_of(a[1], kElem[type], 3), *v = rows_of(a[2], kElem[type], 3);
    if (!k || !v || !same_shape(*k, *v) || k->device() != c.k->device() || k->size(1) != c.H_kv || k->size(2) != c.D ||
        !stream_of(a[10], k->device(), false, stream))
        Py_RETURN_NONE;
    const long long strides[4] = {stride_of(*k, 0), stride_of(*k, 1), stride_of(*v, 0), stride_of(*v, 1)};
    const int rc = launch(k->device(), [&] {
        return g_write[type](k->data_ptr(), v->data_ptr(), strides, c.k->data_ptr(), c.v->data_ptr(), c.k_scale, c.v_scale,
                             (const int *)c.table->data_ptr(), (const int *)c.start->data_ptr(), (const int *)c.kv_len->data_ptr(),
                             c.kind, (int)k->size(0), c.B, c.H_kv, c.D, c.n_pages, c.page, c.width, stream);
    });
    return rc ? PyLong_FromLong(rc) : PyTuple_Pack(2, a[3], a[4]);
    END_HANDLE_TH_ERRORS
}

// read(type, k_pages, v_pages, page_table, start, kv_len, n_rows, k_scale, v_scale, k, v, stream) -> (k, v)
PyObject *py_read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const int type = n == 12 ? type_of(a[0]) : 0;
    Cache c;
    void *stream;
    int T;
    at::Tensor k, v;
    if (n != 12 || !g_read[type] || !cache_of(a + 1, a[7], a[8], kElem[type], c) || !int_of(a[6], T) || T < 1 ||
        !stream_of(a[11], c.k->device(), any_none(a + 9, 2), stream))
        Py_RETURN_NONE;
    const int64_t shape[3] = {T, c.H_kv, c.D};
    if (!rows_output(a[9], *c.k, shape, kElem[type], k) || !rows_output(a[10], *c.k, shape, kElem[type], v))
        Py_RETURN_NONE;
    const long long strides[4] = {stride_of(k, 0), stride_of(k, 1), stride_of(v, 0), stride_of(v, 1)};
    const int rc = launch(c.k->device(), [&] {
        return g_read[type](k.data_ptr(), v.data_ptr(), strides, c.k->data_ptr(), c.v->data_ptr(), c.k_scale, c.v_scale,
                            (const int *)c.table->data_ptr(), (const int *)c.start->data_ptr(), (const int *)c.kv_len->data_ptr(),
                            c.kind, T, c.B, c.H_kv, c.D, c.n_pages, c.page, c.width, stream);
    });
    return rc ? PyLong_FromLong(rc) : pack({&k, &v});
    END_HANDLE_TH_ERRORS
}

// paged(type, q, k_pages, v_pages, page_table, start, kv_len, k_scale, v_scale, o, lse, workspace, causal, scale, max_q, stream)
// -> (o, lse)
PyObject *py_paged(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const int type = n == 16 ? type_of(a[0]) : 0, causal = n == 16 ? truth(a[12]) : -1;
    Cache c;
    void *stream;
    float scale;
    at::Tensor o, lse, ws;
    if (n != 16 || causal < 0 || !g_paged[type] || !g_paged_ws || !cache_of(a + 2, a[7], a[8], kElem[type], c) ||
        !scale_of(a[13], c.D, scale))
        Py_RETURN_NONE;
    const at::Tensor *q = rows_of(a[1], kElem[type], 3);
    if (!q || q->device() != c.k->device() || q->size(2) != c.D || q->size(1) % c.H_kv ||
        !stream_of(a[15], c.k->device(), any_none(a + 9, 3), stream))
        Py_RETURN_NONE;
    const int T = (int)q->size(0), H_q = (int)q->size(1);
    int max_q = T;
    if (a[14] != Py_None && !int_of(a[14], max_q))
        Py_RETURN_NONE;
    const long long need = g_paged_ws(T, c.B, H_q, c.H_kv, c.D);
    if (need < 1)
        Py_RETURN_NONE;
    if (a[11] != Py_None) {
        if (!THPVariable_CheckExact(a[11]))
            Py_RETURN_NONE;
        ws = THPVariable_Unpack(a[11]);
        if (!plain(a[11], ws.scalar_type(), 0) || ws.device() != q->device())
            Py_RETURN_NONE;
    }
    const int64_t o_shape[3] = {T, H_q, c.D}, lse_shape[2] = {T, H_q};
    if (!rows_output(a[9], *q, o_shape, kElem[type], o) || !o.is_contiguous() ||
        !rows_output(a[10], *q, lse_shape, at::kFloat, lse) || !lse.is_contiguous())
        Py_RETURN_NONE;
    if (!ws.defined())
        ws = allocate([&] { return at::empty({need}, q->options().dtype(at::kByte)); });
    const long long strides[2] = {stride_of(*q, 0), stride_of(*q, 1)};
    const int rc = launch(q->device(), [&] {
        return g_paged[type](q->data_ptr(), strides, o.data_ptr(), (float *)lse.data_ptr(), c.k->data_ptr(), c.v->data_ptr(),
                             c.k_scale, c.v_scale, (const int *)c.table->data_ptr(), (const int *)c.start->data_ptr(),
                             (const int *)c.kv_len->data_ptr(), c.kind, ws.data_ptr(), (long long)ws.nbytes(), max_q, T, c.B, H_q,
                             c.H_kv, c.D, c.n_pages, c.page, c.width, causal, scale, stream);
    });
    return rc ? PyLong_FromLong(rc) : pack({&o, &lse});
    END_HANDLE_TH_ERRORS
}

// set_serving_entries(addresses of rope, cache_write, cache_read and paged_fwd, bf16 and fp16 of each, and of the last one's
// workspace size)
PyObject *py_set_serving_entries(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[9];
    if (n != 9) {
        PyErr_SetString(PyExc_TypeError, "set_serving_entries takes nine addresses");
        return nullptr;
    }
    for (int i = 0; i < 9; ++i)
        p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred())
        return nullptr;
    for (int i = 0; i < 2; ++i) {
        g_rope[i] = (RopeFn)p[i];
        g_write[i] = (WriteFn)p[2 + i];
        g_read[i] = (ReadFn)p[4 + i];
        g_paged[i] = (PagedFn)p[6 + i];
    }
    g_paged_ws = (PagedWsFn)p[8];
    Py_RETURN_NONE;
}

// set_entries(addresses of fwd bf16, fwd fp16, splitkv bf16, splitkv fp16, bwd bf16, bwd fp16, workspace size; then the
// function that returns a device's current stream)
PyObject *py_set_entries(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    void *p[7];
    if (n != 8 || !PyCallable_Check(a[7])) {
        PyErr_SetString(PyExc_TypeError, "set_entries takes seven addresses and a function");
        return nullptr;
    }
    for (int i = 0; i < 7; ++i)
        p[i] = PyLong_AsVoidPtr(a[i]);
    if (PyErr_Occurred())
        return nullptr;
    for (int i = 0; i < 2; ++i) {
        g_fwd[i] = (FwdFn)p[i];
        g_split[i] = (SplitFn)p[2 + i];
        g_bwd[i] = (BwdFn)p[4 + i];
    }
    g_ws = (WsFn)p[6];
    Py_INCREF(a[7]);
    Py_XSETREF(g_current_stream, a[7]);
    Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"fwd", (PyCFunction)(void (*)(void))py_fwd, METH_FASTCALL, nullptr},
    {"splitkv", (PyCFunction)(void (*)(void))py_splitkv, METH_FASTCALL, nullptr},
    {"bwd", (PyCFunction)(void (*)(void))py_bwd, METH_FASTCALL, nullptr},
    {"rope", (PyCFunction)(void (*)(void))py_rope, METH_FASTCALL, nullptr},
    {"write", (PyCFunction)(void (*)(void))py_write, METH_FASTCALL, nullptr},
    {"read", (PyCFunction)(void (*)(void))py_read, METH_FASTCALL, nullptr},
    {"paged", (PyCFunction)(void (*)(void))py_paged, METH_FASTCALL, nullptr},
    {"set_serving_entries", (PyCFunction)(void (*)(void))py_set_serving_entries, METH_FASTCALL, nullptr},
    {"set_entries", (PyCFunction)(void (*)(void))py_set_entries, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&kModule); }

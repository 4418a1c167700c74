// Python binding of librkblock (rk_block.h): argument marshalling only, as the module _rkblock
// that block.py wraps.
//
// The smallest calls take the GPU 3 to 6 us, and a launch costs the host 4; marshalling in Python added
// 5 to 8 more a call.  So tensors are looked at, outputs and workspaces allocated (torch's allocator) and pointers handed on
// here.  Whatever the C call cannot take is refused with block.RKBError, as are its non-OK codes.
#include <Python.h>
#include <hip/hip_runtime_api.h>

#include <cmath>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "rk_block.h"

namespace {

PyObject *g_error = nullptr, *g_ckpt = nullptr, *g_kv8 = nullptr, *g_bias = nullptr;  // block.RKBError, Ckpt8, Kv8, RelBias
PyObject *n_codes, *n_exps, *n_dtype, *n_shape, *n_table, *n_max_distance, *n_two_sided;  // attribute names
PyObject *g_dtypes[3];                              // torch.float32, float16, bfloat16 by RKB_F32 ..

struct refused {};  // thrown within this file once the Python error is set

[[noreturn]] void fail(int code, const char *where, const char *why = nullptr)
{
    PyObject *text = why ? PyUnicode_FromFormat("%s (%s)", where, why) : PyUnicode_FromString(where);
    PyObject *err = text ? PyObject_CallFunction(g_error, "iO", code, text) : nullptr;
    Py_XDECREF(text);
    if (err) {
        PyErr_SetObject(g_error, err);
        Py_DECREF(err);
    }
    throw refused();
}

void check(int rc, const char *where)
{
    if (rc != RKB_OK) fail(rc, where);
}

int dtype_of(const at::Tensor &t, const char *where, bool half_only = false)
{
    switch (t.scalar_type()) {
    case at::kHalf: return RKB_F16;
    case at::kBFloat16: return RKB_BF16;
    case at::kFloat:
        if (!half_only) return RKB_F32;
        [[fallthrough]];
    default: fail(RKB_E_INVAL, where, "type");
    }
}

const at::Tensor &tensor(PyObject *o, const char *where)
{
    if (!THPVariable_Check(o)) fail(RKB_E_INVAL, where, "not a tensor of the GPU");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) fail(RKB_E_INVAL, where, "not a tensor of the GPU");
    return t;
}

// A tensor as a matrix: leading dimensions count as rows, which must be evenly spaced.
struct matrix {
    void *p;
    int64_t rows, cols, stride;
    bool aligned() const { return (uintptr_t)p % 16 == 0 && (rows <= 1 || (stride % 8 == 0 && stride <= (int64_t)1 << 22)); }
};

matrix as_matrix(const at::Tensor &t, const char *where)
{
    const int64_t dims = t.dim();
    if (dims == 0) fail(RKB_E_INVAL, where, "no columns");
    matrix m{t.data_ptr(), 1, t.size(dims - 1), t.size(dims - 1)};
    for (int64_t i = dims - 2; i >= 0; --i) m.rows *= t.size(i);
    if (m.rows == 0) return m;  // no row, so none that is out of place
    int64_t next = -1;  // what the next outer dimension's stride has to be
    for (int64_t i = dims - 2; i >= 0; --i) {
        const int64_t n = t.size(i);
        if (n == 1) continue;
        if (next < 0)
            m.stride = t.stride(i);
        else if (t.stride(i) != next)
            fail(RKB_E_INVAL, where, "rows that are not evenly spaced");
        next = t.stride(i) * n;
    }
    if (m.cols > 1 && t.stride(dims - 1) != 1) fail(RKB_E_INVAL, where, "columns that are not adjacent");
    return m;
}

// The same of a tensor that goes with another one: of its device, of type `type`, and of the sizes given (-1: any).
matrix as_matrix(PyObject *o, const char *where, const at::Tensor &like, at::ScalarType type, int64_t rows, int64_t cols)
{
    const at::Tensor &t = tensor(o, where);
    if (t.scalar_type() != type || t.get_device() != like.get_device()) fail(RKB_E_INVAL, where, "types or devices differ");
    const matrix m = as_matrix(t, where);
    if ((rows >= 0 && m.rows != rows) || (cols >= 0 && m.cols != cols)) fail(RKB_E_INVAL, where, "sizes do not match");
    return m;
}

// A contiguous vector of n elements, or NULL for None.
void *as_vector(PyObject *o, const char *where, const at::Tensor &like, at::ScalarType type, int64_t n)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, where);
    if (t.scalar_type() != type || t.get_device() != like.get_device()) fail(RKB_E_INVAL, where, "types or devices differ");
    if (t.numel() != n || !t.is_contiguous()) fail(RKB_E_INVAL, where, "sizes do not match");
    return t.data_ptr();
}

struct owned {  // a new reference
    PyObject *o;
    explicit owned(PyObject *p) : o(p)
    {
        if (!p) throw refused();
    }
    ~owned() { Py_XDECREF(o); }
    owned(const owned &) = delete;
    PyObject *release()
    {
        PyObject *p = o;
        o = nullptr;
        return p;
    }
};

bool is_ckpt(PyObject *o) { return PyObject_TypeCheck(o, (PyTypeObject *)g_ckpt); }

struct ckpt {
    const int8_t *codes = nullptr;
    const uint8_t *exps = nullptr;
};

// A Ckpt8 of a [rows, cols] matrix of type `type`.
ckpt as_ckpt(PyObject *o, const char *where, const at::Tensor *like, int type, int64_t rows, int64_t cols)
{
    owned codes(PyObject_GetAttr(o, n_codes)), exps(PyObject_GetAttr(o, n_exps)), dtype(PyObject_GetAttr(o, n_dtype));
    const at::Tensor &c = tensor(codes.o, where), &e = tensor(exps.o, where);
    const int64_t groups = (cols + RKB_GROUP - 1) / RKB_GROUP;
    if (dtype.o != g_dtypes[type] || c.scalar_type() != at::kChar || e.scalar_type() != at::kByte ||
        e.get_device() != c.get_device() || (like && like->get_device() != c.get_device()))
        fail(RKB_E_INVAL, where, "types or devices differ");
    if (c.dim() != 2 || e.dim() != 2 || c.size(0) != rows || e.size(0) != rows || c.size(1) != groups * RKB_GROUP ||
        e.size(1) != groups || !c.is_contiguous() || !e.is_contiguous())
        fail(RKB_E_INVAL, where, "sizes do not match");
    return {(const int8_t *)c.data_ptr(), (const uint8_t *)e.data_ptr()};
}

// x of a backward pass: a matrix or its Ckpt8.
struct kept_matrix {
    matrix m{nullptr, 0, 0, 0};
    ckpt c;
};

kept_matrix as_kept(PyObject *o, const char *where, const at::Tensor &like, int type, int64_t rows, int64_t cols)
{
    kept_matrix k;
    if (is_ckpt(o))
        k.c = as_ckpt(o, where, &like, type, rows, cols);
    else
        k.m = as_matrix(o, where, like, like.scalar_type(), rows, cols);
    return k;
}

// A tensor's device as the current one while a call runs, and its current stream.
struct on_device {
    int before = -1;
    void *stream;
    on_device(const at::Tensor &t, const char *where)
    {
        const int want = t.get_device();
        if (hipGetDevice(&before) != hipSuccess) fail(RKB_E_DEVICE, where);
        if (before == want)
            before = -1;
        else if (hipSetDevice(want) != hipSuccess)
            fail(RKB_E_DEVICE, where);
        stream = (void *)c10::hip::getCurrentHIPStream((c10::DeviceIndex)want).stream();
    }
    ~on_device()
    {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

at::Tensor like_of(const at::Tensor &t, at::IntArrayRef shape) { return at::empty(shape, t.options()); }
at::Tensor like_of(const at::Tensor &t, at::IntArrayRef shape, at::ScalarType type) { return at::empty(shape, t.options().dtype(type)); }

struct workspace {
    at::Tensor t;
    void *p = nullptr;
    size_t bytes = 0;
    void need(const at::Tensor &like, size_t n)
    {
        if (n == 0) return;
        t = like_of(like, {(int64_t)n}, at::kByte);
        p = t.data_ptr();
        bytes = n;
    }
};

PyObject *wrap(const at::Tensor &t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}

PyObject *wrap_all(std::initializer_list<const at::Tensor *> ts)
{
    owned out(PyTuple_New((Py_ssize_t)ts.size()));
    Py_ssize_t i = 0;
    for (const at::Tensor *t : ts) PyTuple_SET_ITEM(out.o, i++, owned(wrap(*t)).release());
    return out.release();
}

struct new_ckpt {
    at::Tensor codes, exps;
    new_ckpt(const at::Tensor &like, int64_t rows, int64_t cols)
    {
        const int64_t groups = (cols + RKB_GROUP - 1) / RKB_GROUP;
        codes = like_of(like, {rows, groups * RKB_GROUP}, at::kChar);
        exps = like_of(like, {rows, groups}, at::kByte);
    }
    PyObject *make(PyObject *shape, PyObject *dtype) const
    {
        owned c(wrap(codes)), e(wrap(exps));
        PyObject *args[] = {c.o, e.o, shape, dtype};
        return owned(PyObject_Vectorcall(g_ckpt, args, 4, nullptr)).release();
    }
};

long as_int(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw refused();
    return v;
}

bool as_bool(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw refused();
    return v != 0;
}

// Runs one call's body: refusals and C++ exceptions become Python errors.
template <class F>
PyObject *guarded(Py_ssize_t want, Py_ssize_t got, F body)
{
    HANDLE_TH_ERRORS
    if (want != got) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return body();
    } catch (const refused &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// ------------------------------------------------------------------ the calls

PyObject *layer_norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(4, n, [&] {
        const char *where = "rkb_layer_norm_fwd";
        const at::Tensor &x = tensor(a[0], where);
        const int type = dtype_of(x, where);
        const matrix m = as_matrix(x, where);
        at::ScalarType wt = x.scalar_type();
        if (a[1] != Py_None || a[2] != Py_None) {
            wt = tensor(a[1] != Py_None ? a[1] : a[2], where).scalar_type();
            if (wt != x.scalar_type() && wt != at::kFloat) fail(RKB_E_INVAL, where, "types or devices differ");
        }
        void *w = as_vector(a[1], where, x, wt, m.cols), *b = as_vector(a[2], where, x, wt, m.cols);
        const double eps = PyFloat_AsDouble(a[3]);
        if (eps == -1.0 && PyErr_Occurred()) throw refused();
        const on_device on(x, where);
        const at::Tensor y = like_of(x, x.sizes());
        const at::IntArrayRef lead = x.sizes().slice(0, x.dim() - 1);
        const at::Tensor mean = like_of(x, lead, at::kFloat), rstd = like_of(x, lead, at::kFloat);
        check(rkb_layer_norm_fwd(type, wt == at::kFloat ? RKB_F32 : type, m.rows, m.cols, m.p, m.stride, w, b, (float)eps,
                                 y.data_ptr(), m.cols, (float *)mean.data_ptr(), (float *)rstd.data_ptr(), on.stream), where);
        return wrap_all({&y, &mean, &rstd});
    });
}

PyObject *layer_norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(6, n, [&] {
        const char *where = "rkb_layer_norm_bwd";
        const at::Tensor &dy = tensor(a[0], where);
        const int type = dtype_of(dy, where);
        const matrix m = as_matrix(dy, where);
        const kept_matrix x = as_kept(a[1], where, dy, type, m.rows, m.cols);
        void *mean = as_vector(a[2], where, dy, at::kFloat, m.rows), *rstd = as_vector(a[3], where, dy, at::kFloat, m.rows);
        if (a[2] == Py_None || a[3] == Py_None) fail(RKB_E_INVAL, where, "no mean or rstd");
        at::ScalarType wt = dy.scalar_type();
        if (a[4] != Py_None) {
            wt = tensor(a[4], where).scalar_type();
            if (wt != dy.scalar_type() && wt != at::kFloat) fail(RKB_E_INVAL, where, "types or devices differ");
        }
        void *w = as_vector(a[4], where, dy, wt, m.cols);
        const bool bias = as_bool(a[5]);
        const on_device on(dy, where);
        const at::Tensor dx = like_of(dy, dy.sizes());
        at::Tensor dw, db;
        if (w) dw = like_of(dy, {m.cols}, wt);
        if (bias) db = like_of(dy, {m.cols}, wt);
        workspace ws;
        if (w || bias) {
            size_t bytes = 0;
            check(rkb_layer_norm_bwd_workspace(type, m.rows, m.cols, &bytes), where);
            ws.need(dy, bytes);
        }
        check(rkb_layer_norm_bwd(type, wt == at::kFloat ? RKB_F32 : type, m.rows, m.cols, m.p, m.stride, x.m.p, x.m.stride,
                                 x.c.codes, x.c.exps, (const float *)mean, (const float *)rstd, w, dx.data_ptr(), m.cols,
                                 w ? dw.data_ptr() : nullptr, bias ? db.data_ptr() : nullptr, ws.p, ws.bytes, on.stream), where);
        return wrap_all({&dx, &dw, &db});
    });
}

PyObject *ckpt8_save(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(1, n, [&] {
        const char *where = "rkb_ckpt8_save";
        const at::Tensor &x = tensor(a[0], where);
        const int type = dtype_of(x, where);
        const matrix m = as_matrix(x, where);
        if (m.cols == 0) fail(RKB_E_INVAL, where, "no columns");
        const on_device on(x, where);
        const new_ckpt c(x, m.rows, m.cols);
        check(rkb_ckpt8_save(type, m.rows, m.cols, m.p, m.stride, (int8_t *)c.codes.data_ptr(), (uint8_t *)c.exps.data_ptr(),
                             on.stream), where);
        owned shape(PyObject_GetAttr(a[0], n_shape));
        return c.make(shape.o, g_dtypes[type]);
    });
}

PyObject *ckpt8_load(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(1, n, [&] {
        const char *where = "rkb_ckpt8_load";
        if (!is_ckpt(a[0])) fail(RKB_E_INVAL, where, "not a checkpoint on the GPU");
        owned dtype(PyObject_GetAttr(a[0], n_dtype)), shape(PyObject_GetAttr(a[0], n_shape)), codes(PyObject_GetAttr(a[0], n_codes));
        int type = 0;
        while (type < 3 && g_dtypes[type] != dtype.o) ++type;
        const Py_ssize_t dims = PyTuple_Check(shape.o) ? PyTuple_GET_SIZE(shape.o) : 0;
        if (type == 3 || dims == 0) fail(RKB_E_INVAL, where, "not a checkpoint on the GPU");
        c10::SmallVector<int64_t, 6> sizes;
        int64_t rows = 1;
        for (Py_ssize_t i = 0; i < dims; ++i) {
            sizes.push_back(as_int(PyTuple_GET_ITEM(shape.o, i)));
            if (i + 1 < dims) rows *= sizes.back();
        }
        const at::Tensor &like = tensor(codes.o, where);
        const ckpt c = as_ckpt(a[0], where, nullptr, type, rows, sizes.back());
        const on_device on(like, where);
        const at::ScalarType types[] = {at::kFloat, at::kHalf, at::kBFloat16};
        const at::Tensor x = like_of(like, sizes, types[type]);
        check(rkb_ckpt8_load(type, rows, sizes.back(), c.codes, c.exps, x.data_ptr(), sizes.back(), on.stream), where);
        return wrap(x);
    });
}

PyObject *weight_grad(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(2, n_args, [&] {
        const char *where = "rkb_weight_grad";
        const at::Tensor &dy = tensor(a[0], where);
        const int type = dtype_of(dy, where, true);
        const matrix m = as_matrix(dy, where);
        int64_t k;
        if (is_ckpt(a[1])) {
            owned shape(PyObject_GetAttr(a[1], n_shape));
            const Py_ssize_t dims = PyTuple_Check(shape.o) ? PyTuple_GET_SIZE(shape.o) : 0;
            if (dims == 0) fail(RKB_E_INVAL, where, "sizes do not match");
            k = as_int(PyTuple_GET_ITEM(shape.o, dims - 1));
        } else {
            const at::Tensor &x = tensor(a[1], where);
            if (x.dim() == 0) fail(RKB_E_INVAL, where, "no columns");
            k = x.size(x.dim() - 1);
        }
        const kept_matrix x = as_kept(a[1], where, dy, type, m.rows, k);
        const on_device on(dy, where);
        const at::Tensor dw = like_of(dy, {m.cols, k});
        size_t bytes = 0;
        check(rkb_weight_grad_workspace(type, m.rows, m.cols, k, x.c.codes != nullptr, m.aligned() && (x.c.codes || x.m.aligned()),
                                        &bytes), where);
        workspace ws;
        ws.need(dy, bytes);
        check(rkb_weight_grad(type, m.rows, m.cols, k, m.p, m.stride, x.m.p, x.m.stride, x.c.codes, x.c.exps, dw.data_ptr(), k, ws.p,
                              ws.bytes, on.stream), where);
        return wrap(dw);
    });
}

// x, wg and wu of a gated block.
struct gated_args {
    int type;
    matrix x, wg, wu;
    gated_args(PyObject *const *a, const char *where)
    {
        const at::Tensor &t = tensor(a[0], where);
        type = dtype_of(t, where, true);
        x = as_matrix(t, where);
        wg = as_matrix(a[1], where, t, t.scalar_type(), -1, x.cols);
        wu = as_matrix(a[2], where, t, t.scalar_type(), wg.rows, x.cols);
    }
    bool aligned() const { return x.aligned() && wg.aligned() && wu.aligned() && wg.stride == wu.stride; }
};

PyObject *gated_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(5, n, [&] {
        const char *where = "rkb_gated_fwd";
        const gated_args in(a, where);
        const at::Tensor &x = THPVariable_Unpack(a[0]);
        const int act = (int)as_int(a[3]), keep = (int)as_int(a[4]);
        const int64_t rows = in.x.rows, d = in.x.cols, f = in.wg.rows;
        const on_device on(x, where);
        c10::SmallVector<int64_t, 6> shape(x.sizes().begin(), x.sizes().end());
        shape.back() = f;
        const at::Tensor h = like_of(x, shape);
        at::Tensor g, u;
        std::optional<new_ckpt> g8, u8;
        void *gp = nullptr, *up = nullptr;
        uint8_t *ge = nullptr, *ue = nullptr;
        if (keep == RKB_KEEP_FULL || keep == RKB_KEEP_16BIT) {
            const at::ScalarType t = keep == RKB_KEEP_FULL ? at::kFloat : x.scalar_type();
            g = like_of(x, shape, t);
            u = like_of(x, shape, t);
            gp = g.data_ptr();
            up = u.data_ptr();
        } else if (keep == RKB_KEEP_8BIT) {
            g8.emplace(x, rows, f);
            u8.emplace(x, rows, f);
            gp = g8->codes.data_ptr();
            up = u8->codes.data_ptr();
            ge = (uint8_t *)g8->exps.data_ptr();
            ue = (uint8_t *)u8->exps.data_ptr();
        }
        size_t bytes = 0;
        check(rkb_gated_fwd_workspace(in.type, rows, d, f, in.aligned(), &bytes), where);
        workspace ws;
        ws.need(x, bytes);
        check(rkb_gated_fwd(in.type, act, keep, rows, d, f, in.x.p, in.x.stride, in.wg.p, in.wg.stride, in.wu.p, in.wu.stride,
                            h.data_ptr(), f, gp, up, ge, ue, ws.p, ws.bytes, on.stream), where);
        owned out(PyTuple_New(2));
        PyTuple_SET_ITEM(out.o, 0, owned(wrap(h)).release());
        if (g8) {
            owned size(PyTuple_New((Py_ssize_t)shape.size())), both(PyTuple_New(2));
            for (size_t i = 0; i < shape.size(); ++i)
                PyTuple_SET_ITEM(size.o, (Py_ssize_t)i, owned(PyLong_FromLongLong(shape[i])).release());
            PyTuple_SET_ITEM(both.o, 0, g8->make(size.o, g_dtypes[RKB_F32]));
            PyTuple_SET_ITEM(both.o, 1, u8->make(size.o, g_dtypes[RKB_F32]));
            PyTuple_SET_ITEM(out.o, 1, both.release());
        } else if (g.defined()) {
            PyTuple_SET_ITEM(out.o, 1, wrap_all({&g, &u}));
        } else {
            Py_INCREF(Py_None);
            PyTuple_SET_ITEM(out.o, 1, Py_None);
        }
        return out.release();
    });
}

PyObject *gated_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(7, n, [&] {
        const char *where = "rkb_gated_bwd";
        const gated_args in(a + 1, where);
        const at::Tensor &x = THPVariable_Unpack(a[1]);
        const int64_t rows = in.x.rows, d = in.x.cols, f = in.wg.rows;
        const matrix dh = as_matrix(a[0], where, x, x.scalar_type(), rows, f);
        const int act = (int)as_int(a[4]);
        int keep = RKB_KEEP_NONE;
        const void *g = nullptr, *u = nullptr;
        ckpt g8, u8;
        if (a[5] != Py_None) {
            if (!PyTuple_Check(a[5]) || PyTuple_GET_SIZE(a[5]) != 2) fail(RKB_E_INVAL, where, "kept");
            PyObject *go = PyTuple_GET_ITEM(a[5], 0), *uo = PyTuple_GET_ITEM(a[5], 1);
            if (is_ckpt(go) && is_ckpt(uo)) {
                keep = RKB_KEEP_8BIT;
                g8 = as_ckpt(go, where, &x, RKB_F32, rows, f);
                u8 = as_ckpt(uo, where, &x, RKB_F32, rows, f);
                g = g8.codes;
                u = u8.codes;
            } else {
                const bool full = tensor(go, where).scalar_type() == at::kFloat;
                keep = full ? RKB_KEEP_FULL : RKB_KEEP_16BIT;
                const at::ScalarType t = full ? at::kFloat : x.scalar_type();
                const matrix gm = as_matrix(go, where, x, t, rows, f), um = as_matrix(uo, where, x, t, rows, f);
                if (rows > 1 && (gm.stride != f || um.stride != f)) fail(RKB_E_INVAL, where, "g and u are not contiguous");
                g = gm.p;
                u = um.p;
            }
        }
        const bool want_h = as_bool(a[6]);
        const on_device on(x, where);
        const at::Tensor dx = like_of(x, x.sizes()), dwg = like_of(x, {f, d}), dwu = like_of(x, {f, d});
        at::Tensor h;
        if (want_h) {
            c10::SmallVector<int64_t, 6> shape(x.sizes().begin(), x.sizes().end());
            shape.back() = f;
            h = like_of(x, shape);
        }
        size_t bytes = 0;
        check(rkb_gated_bwd_workspace(in.type, keep, rows, d, f, in.aligned(), &bytes), where);
        workspace ws;
        ws.need(x, bytes);
        check(rkb_gated_bwd(in.type, act, keep, rows, d, f, dh.p, dh.stride, in.x.p, in.x.stride, in.wg.p, in.wg.stride, in.wu.p,
                            in.wu.stride, g, u, g8.exps, u8.exps, dx.data_ptr(), d, dwg.data_ptr(), dwu.data_ptr(), d,
                            want_h ? h.data_ptr() : nullptr, f, ws.p, ws.bytes, on.stream), where);
        return wrap_all({&dx, &dwg, &dwu, &h});
    });
}

// ------------------------------------------------------------------ attention

// A [batch, rows, heads, dim] tensor that goes with another one: of its device, of type `type`, and of the sizes given (-1: any).
rkb_heads as_heads(const at::Tensor &t, const char *where, const at::Tensor &like, at::ScalarType type, int64_t batch, int64_t rows,
                   int64_t heads, int64_t dim)
{
    if (t.scalar_type() != type || t.get_device() != like.get_device()) fail(RKB_E_INVAL, where, "types or devices differ");
    if (t.dim() != 4 || (batch >= 0 && t.size(0) != batch) || (rows >= 0 && t.size(1) != rows) || (heads >= 0 && t.size(2) != heads) ||
        (dim >= 0 && t.size(3) != dim))
        fail(RKB_E_INVAL, where, "sizes do not match");
    if (t.size(3) > 1 && t.stride(3) != 1) fail(RKB_E_INVAL, where, "columns that are not adjacent");
    return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}

bool aligned(const at::Tensor &t, const rkb_heads &h)
{
    auto good = [&](int i, int64_t s) { return t.size(i) <= 1 || s % 8 == 0; };
    return (uintptr_t)h.p % 16 == 0 && good(0, h.batch) && good(1, h.row) && good(2, h.head) && (t.size(1) <= 1 || h.row <= (int64_t)1 << 22);
}

// None, or a contiguous int32 tensor with one element per sequence.
const int32_t *as_counts(PyObject *o, const char *where, const at::Tensor &like, int64_t batch)
{
    return (const int32_t *)as_vector(o, where, like, at::kInt, batch);
}

// An int, or a tensor of an int32 per sequence.
void as_first(PyObject *o, const char *where, const at::Tensor &like, int64_t batch, int64_t *first, const int32_t **firsts)
{
    *first = 0;
    *firsts = nullptr;
    if (THPVariable_Check(o))
        *firsts = as_counts(o, where, like, batch);
    else
        *first = as_int(o);
}

struct kv8 {
    rkb_kv8 c;
    int64_t batch, tokens, heads, dim;
    int type;
    const at::Tensor *codes;
};

kv8 as_kv8(PyObject *o, const char *where, const at::Tensor *like)
{
    owned codes(PyObject_GetAttr(o, n_codes)), exps(PyObject_GetAttr(o, n_exps)), dtype(PyObject_GetAttr(o, n_dtype)), shape(PyObject_GetAttr(o, n_shape));
    const at::Tensor &c = tensor(codes.o, where), &e = tensor(exps.o, where);
    kv8 k{};
    while (k.type < 3 && g_dtypes[k.type] != dtype.o) ++k.type;
    if ((k.type != RKB_F16 && k.type != RKB_BF16) || c.scalar_type() != at::kChar || e.scalar_type() != at::kByte ||
        e.get_device() != c.get_device() || (like && like->get_device() != c.get_device()))
        fail(RKB_E_INVAL, where, "types or devices differ");
    if (!PyTuple_Check(shape.o) || PyTuple_GET_SIZE(shape.o) != 4) fail(RKB_E_INVAL, where, "sizes do not match");
    int64_t *const to[] = {&k.batch, &k.tokens, &k.heads, &k.dim};
    for (int i = 0; i < 4; ++i) {
        *to[i] = as_int(PyTuple_GET_ITEM(shape.o, i));
        if (*to[i] < 0 || *to[i] > RKB_MAX_TOKENS) fail(RKB_E_INVAL, where, "sizes do not match");
    }
    const int64_t blocks = (k.tokens + RKB_GROUP - 1) / RKB_GROUP, ld = (k.dim + 15) / 16 * 16;
    if (c.sizes() != at::IntArrayRef({2, k.batch, k.heads, blocks * RKB_GROUP, ld}) || e.sizes() != at::IntArrayRef({2, k.batch, k.heads, blocks}) ||
        !c.is_contiguous() || !e.is_contiguous())
        fail(RKB_E_INVAL, where, "sizes do not match");
    k.c = {(int8_t *)c.data_ptr(), (uint8_t *)e.data_ptr(), k.tokens};
    k.codes = &THPVariable_Unpack(codes.o);  // the cache object holds it while the call runs
    return k;
}

// scale, lens, mask, causal, first and bias: a[0] .. a[5].
struct attn_args {
    rkb_attn a{};
    const at::Tensor *table = nullptr;
    attn_args(PyObject *const *o, const char *where, const at::Tensor &q, int64_t k_rows, int64_t kv_heads)
    {
        a.dtype = dtype_of(q, where, true);
        a.batch = q.size(0);
        a.q_rows = q.size(1);
        a.k_rows = k_rows;
        a.heads = q.size(2);
        a.kv_heads = kv_heads;
        a.dim = q.size(3);
        if (o[0] == Py_None) {
            a.scale = a.dim > 0 ? (float)(1.0 / std::sqrt((double)a.dim)) : 1.0f;
        } else {
            const double s = PyFloat_AsDouble(o[0]);
            if (s == -1.0 && PyErr_Occurred()) throw refused();
            a.scale = (float)s;
        }
        a.lens = as_counts(o[1], where, q, a.batch);
        if (o[2] != Py_None) {
            const at::Tensor &m = tensor(o[2], where);
            if ((m.scalar_type() != at::kBool && m.scalar_type() != at::kByte) || m.get_device() != q.get_device())
                fail(RKB_E_INVAL, where, "types or devices differ");
            if (m.dim() != 2 || m.size(0) != a.batch || m.size(1) != k_rows) fail(RKB_E_INVAL, where, "sizes do not match");
            if (k_rows > 1 && m.stride(1) != 1) fail(RKB_E_INVAL, where, "columns that are not adjacent");
            a.mask = (const uint8_t *)m.data_ptr();
            a.mask_stride = m.stride(0);
        }
        a.causal = as_bool(o[3]);
        as_first(o[4], where, q, a.batch, &a.first, &a.firsts);
        if (o[5] != Py_None) {
            if (!PyObject_TypeCheck(o[5], (PyTypeObject *)g_bias)) fail(RKB_E_INVAL, where, "bias");
            owned t(PyObject_GetAttr(o[5], n_table)), far(PyObject_GetAttr(o[5], n_max_distance)), two(PyObject_GetAttr(o[5], n_two_sided));
            table = &tensor(t.o, where);
            if ((table->scalar_type() != q.scalar_type() && table->scalar_type() != at::kFloat) || table->get_device() != q.get_device())
                fail(RKB_E_INVAL, where, "types or devices differ");
            if (table->dim() != 2 || table->size(1) != a.heads || table->size(0) > RKB_MAX_BUCKETS || !table->is_contiguous())
                fail(RKB_E_INVAL, where, "sizes do not match");
            const long most = as_int(far.o);
            if (most < 0 || most > RKB_MAX_DISTANCE) fail(RKB_E_INVAL, where, "max_distance");
            a.table = table->data_ptr();
            a.table_dtype = dtype_of(*table, where);
            a.buckets = (int)table->size(0);
            a.max_distance = (int)most;
            a.two_sided = as_bool(two.o);
            if (a.buckets == 0) fail(RKB_E_INVAL, where, "sizes do not match");
        }
    }
};

rkb_heads heads_of(const at::Tensor &t)
{
    if (!t.defined()) return {nullptr, 0, 0, 0};
    return {t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)};
}

// attn_fwd(q, k or cache, v, scale, lens, mask, causal, first, bias, keep)
PyObject *attn_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(10, n, [&] {
        const char *where = "rkb_attn_fwd";
        const at::Tensor &q = tensor(a[0], where);
        const int type = dtype_of(q, where, true);
        const rkb_heads qh = as_heads(q, where, q, q.scalar_type(), -1, -1, -1, -1);
        const bool cached = PyObject_TypeCheck(a[1], (PyTypeObject *)g_kv8);
        kv8 cache{};
        rkb_heads kh{}, vh{};
        int64_t tokens, heads;
        bool fits = aligned(q, qh);
        if (cached) {
            if (a[2] != Py_None) fail(RKB_E_INVAL, where, "a cache and values");
            cache = as_kv8(a[1], where, &q);
            if (cache.type != type || cache.batch != q.size(0) || cache.dim != q.size(3)) fail(RKB_E_INVAL, where, "sizes do not match");
            tokens = cache.tokens;
            heads = cache.heads;
        } else {
            const at::Tensor &k = tensor(a[1], where), &v = tensor(a[2], where);
            kh = as_heads(k, where, q, q.scalar_type(), q.size(0), -1, -1, q.size(3));
            tokens = k.size(1);
            heads = k.size(2);
            vh = as_heads(v, where, q, q.scalar_type(), q.size(0), tokens, heads, q.size(3));
            fits = fits && aligned(k, kh) && aligned(v, vh);
        }
        const attn_args args(a + 3, where, q, tokens, heads);
        const long keep = as_int(a[9]);
        const on_device on(q, where);
        const at::Tensor o = like_of(q, q.sizes());
        at::Tensor o32, lse;
        if (keep != RKB_KEEP_NONE) lse = like_of(q, {q.size(0), q.size(2), q.size(1)}, at::kFloat);
        if (keep == RKB_KEEP_FULL) o32 = like_of(q, q.sizes(), at::kFloat);
        size_t bytes = 0;
        check(rkb_attn_fwd_workspace(&args.a, cached, fits, &bytes), where);
        workspace ws;
        ws.need(q, bytes);
        const rkb_heads oh = heads_of(o);
        check(rkb_attn_fwd(&args.a, &qh, cached ? nullptr : &kh, cached ? nullptr : &vh, cached ? &cache.c : nullptr, &oh,
                           o32.defined() ? (float *)o32.data_ptr() : nullptr, lse.defined() ? (float *)lse.data_ptr() : nullptr, ws.p, ws.bytes,
                           on.stream), where);
        owned out(PyTuple_New(2));
        PyTuple_SET_ITEM(out.o, 0, owned(wrap(o)).release());
        if (lse.defined()) {
            PyTuple_SET_ITEM(out.o, 1, wrap_all({o32.defined() ? &o32 : &o, &lse}));
        } else {
            Py_INCREF(Py_None);
            PyTuple_SET_ITEM(out.o, 1, Py_None);
        }
        return out.release();
    });
}

// attn_bwd(do, q, k, v, kept, scale, lens, mask, causal, first, bias)
PyObject *attn_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(11, n, [&] {
        const char *where = "rkb_attn_bwd";
        const at::Tensor &q = tensor(a[1], where);
        dtype_of(q, where, true);
        const rkb_heads qh = as_heads(q, where, q, q.scalar_type(), -1, -1, -1, -1);
        const at::Tensor &d = tensor(a[0], where), &k = tensor(a[2], where), &v = tensor(a[3], where);
        const rkb_heads dh = as_heads(d, where, q, q.scalar_type(), q.size(0), q.size(1), q.size(2), q.size(3));
        const rkb_heads kh = as_heads(k, where, q, q.scalar_type(), q.size(0), -1, -1, q.size(3));
        const rkb_heads vh = as_heads(v, where, q, q.scalar_type(), q.size(0), k.size(1), k.size(2), q.size(3));
        const attn_args args(a + 5, where, q, k.size(1), k.size(2));
        rkb_heads oh{};
        const float *o32 = nullptr, *lse = nullptr;
        if (a[4] != Py_None) {
            if (!PyTuple_Check(a[4]) || PyTuple_GET_SIZE(a[4]) != 2) fail(RKB_E_INVAL, where, "kept");
            const at::Tensor &o = tensor(PyTuple_GET_ITEM(a[4], 0), where), &l = tensor(PyTuple_GET_ITEM(a[4], 1), where);
            const bool full = o.scalar_type() == at::kFloat;
            oh = as_heads(o, where, q, full ? at::kFloat : q.scalar_type(), q.size(0), q.size(1), q.size(2), q.size(3));
            if (l.scalar_type() != at::kFloat || l.get_device() != q.get_device() || l.sizes() != at::IntArrayRef({q.size(0), q.size(2), q.size(1)}) ||
                !l.is_contiguous() || (full && !o.is_contiguous()))
                fail(RKB_E_INVAL, where, "kept");
            if (full) {
                o32 = (const float *)oh.p;
                oh.p = nullptr;
            }
            lse = (const float *)l.data_ptr();
        }
        const on_device on(q, where);
        const at::Tensor dq = like_of(q, q.sizes()), dk = like_of(k, k.sizes()), dv = like_of(v, v.sizes());
        at::Tensor dtable;
        if (args.table) dtable = like_of(*args.table, args.table->sizes());
        const bool again = a[4] == Py_None, fits = aligned(q, qh) && aligned(d, dh) && aligned(k, kh) && aligned(v, vh);
        size_t bytes = 0;
        check(rkb_attn_bwd_workspace(&args.a, again, fits, &bytes), where);
        workspace ws;
        ws.need(q, bytes);
        // an empty tensor may have no memory at all
        static const float nothing = 0.0f;
        if (!again && !lse) lse = &nothing;
        const rkb_heads dqh = heads_of(dq), dkh = heads_of(dk), dvh = heads_of(dv);
        check(rkb_attn_bwd(&args.a, &dh, &qh, &kh, &vh, &oh, o32, lse, &dqh, &dkh, &dvh, dtable.defined() ? dtable.data_ptr() : nullptr, ws.p,
                           ws.bytes, on.stream), where);
        return wrap_all({&dq, &dk, &dv, &dtable});
    });
}

// kv8_write(cache, k, v, first, counts)
PyObject *kv8_write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(5, n, [&] {
        const char *where = "rkb_kv8_write";
        if (!PyObject_TypeCheck(a[0], (PyTypeObject *)g_kv8)) fail(RKB_E_INVAL, where, "not a cache on the GPU");
        const at::Tensor &k = tensor(a[1], where), &v = tensor(a[2], where);
        const kv8 c = as_kv8(a[0], where, &k);
        if (dtype_of(k, where, true) != c.type) fail(RKB_E_INVAL, where, "types or devices differ");
        const rkb_heads kh = as_heads(k, where, k, k.scalar_type(), c.batch, -1, c.heads, c.dim);
        const rkb_heads vh = as_heads(v, where, k, k.scalar_type(), c.batch, k.size(1), c.heads, c.dim);
        int64_t first;
        const int32_t *firsts;
        as_first(a[3], where, k, c.batch, &first, &firsts);
        const int32_t *counts = as_counts(a[4], where, k, c.batch);
        const on_device on(k, where);
        check(rkb_kv8_write(c.type, c.batch, k.size(1), c.heads, c.dim, &kh, &vh, first, firsts, counts, &c.c, on.stream), where);
        Py_RETURN_NONE;
    });
}

PyObject *kv8_load(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(1, n, [&] {
        const char *where = "rkb_kv8_load";
        if (!PyObject_TypeCheck(a[0], (PyTypeObject *)g_kv8)) fail(RKB_E_INVAL, where, "not a cache on the GPU");
        const kv8 c = as_kv8(a[0], where, nullptr);
        const on_device on(*c.codes, where);
        const at::ScalarType type = c.type == RKB_F16 ? at::kHalf : at::kBFloat16;
        const at::Tensor k = like_of(*c.codes, {c.batch, c.tokens, c.heads, c.dim}, type), v = like_of(k, k.sizes());
        const rkb_heads kh = heads_of(k), vh = heads_of(v);
        check(rkb_kv8_load(c.type, c.batch, c.heads, c.dim, &c.c, &kh, &vh, on.stream), where);
        return wrap_all({&k, &v});
    });
}

// init(RKBError, Ckpt8, (float32, float16, bfloat16), Kv8, RelBias)
PyObject *init(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 5 || !PyTuple_Check(a[2]) || PyTuple_GET_SIZE(a[2]) != 3) {
        PyErr_SetString(PyExc_TypeError, "init(RKBError, Ckpt8, dtypes, Kv8, RelBias)");
        return nullptr;
    }
    Py_INCREF(a[0]);
    Py_INCREF(a[1]);
    Py_INCREF(a[3]);
    Py_INCREF(a[4]);
    g_error = a[0];
    g_ckpt = a[1];
    g_kv8 = a[3];
    g_bias = a[4];
    for (int i = 0; i < 3; ++i) {
        g_dtypes[i] = PyTuple_GET_ITEM(a[2], i);
        Py_INCREF(g_dtypes[i]);
    }
    n_codes = PyUnicode_InternFromString("codes");
    n_exps = PyUnicode_InternFromString("exps");
    n_dtype = PyUnicode_InternFromString("dtype");
    n_shape = PyUnicode_InternFromString("shape");
    n_table = PyUnicode_InternFromString("table");
    n_max_distance = PyUnicode_InternFromString("max_distance");
    n_two_sided = PyUnicode_InternFromString("two_sided");
    Py_RETURN_NONE;
}

#define RKB_CALL(name) {#name, (PyCFunction)(void *)name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {RKB_CALL(init),        RKB_CALL(layer_norm_fwd), RKB_CALL(layer_norm_bwd), RKB_CALL(ckpt8_save),
                         RKB_CALL(ckpt8_load),  RKB_CALL(weight_grad),    RKB_CALL(gated_fwd),      RKB_CALL(gated_bwd),
                         RKB_CALL(attn_fwd),    RKB_CALL(attn_bwd),       RKB_CALL(kv8_write),      RKB_CALL(kv8_load),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rkblock", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__rkblock() { return PyModule_Create(&module); }

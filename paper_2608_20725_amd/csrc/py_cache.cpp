// Python binding of rotary positions and the paged cache (seq_cache.py): checks
// of shapes, types and devices, allocation of results, and the call into the C
// interface on the current stream of the tensors' device.
//
// These calls are small in serving (a new token of each sequence): marshalled
// in Python, as the other operators are, a call took 4 to 8 us beside the 4 of
// the C call, and attention's three allocations another 5.
#include <Python.h>

#include <ATen/core/LegacyTypeDispatch.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <math.h>

#include "im2win_seq.h"

namespace {

PyObject *g_error;  // Im2winError(status, what)

template <class... A>
[[noreturn]] void refuse(PyObject *type, const char *format, A... a)
{
    PyErr_Format(type, format, a...);
    throw python_error();
}

void check(int64_t rc, const char *what)
{
    if (rc >= 0)
        return;
    PyObject *const args = Py_BuildValue("(Ls)", (long long)rc, what);
    if (args) {
        PyErr_SetObject(g_error, args);
        Py_DECREF(args);
    }
    throw python_error();
}

// ---- arguments ----

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o))
        refuse(PyExc_TypeError, "%s must be a tensor", name);
    return THPVariable_Unpack(o);
}

double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1 && PyErr_Occurred())
        throw python_error();
    return v;
}

bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0)
        throw python_error();
    return v != 0;
}

int code(at::ScalarType t)
{
    switch (t) {
    case at::kFloat: return IM2WIN_F32;
    case at::kHalf: return IM2WIN_F16;
    case at::kBFloat16: return IM2WIN_BF16;
    case at::kChar: return SEQ_I8;
    case at::kFloat8_e4m3fn: return SEQ_E4M3;
    default: refuse(PyExc_ValueError, "no operator here takes elements of type %s", c10::toString(t));
    }
}
bool coded(int dt) { return dt == SEQ_I8 || dt == SEQ_E4M3; }

void on_device(const at::Tensor &t, c10::Device d)
{
    if (t.device() != d)
        refuse(PyExc_ValueError, "all tensors must be on %s", d.str().c_str());
}

void dense_channels(const at::Tensor &t, const char *name)
{
    const int64_t last = t.dim() - 1;
    if (t.size(last) > 1 && t.stride(last) != 1)
        refuse(PyExc_ValueError, "%s must be dense in its last dimension", name);
}

void like(const at::Tensor &t, const at::Tensor &x, const char *name)
{
    if (t.sizes() != x.sizes() || t.scalar_type() != x.scalar_type())
        refuse(PyExc_ValueError, "%s must have the shape and type of the operand", name);
    on_device(t, x.device());
    dense_channels(t, name);
}

// A contiguous int32 [B] tensor, or None: null.
const int32_t *counts(PyObject *o, const char *name, int64_t B, c10::Device d)
{
    if (o == Py_None)
        return nullptr;
    const at::Tensor &t = tensor(o, name);
    if (t.scalar_type() != at::kInt || t.dim() != 1 || t.size(0) != B || !t.is_contiguous())
        refuse(PyExc_ValueError, "%s must be a contiguous int32 [%lld] tensor", name, (long long)B);
    on_device(t, d);
    return (const int32_t *)t.const_data_ptr();
}

void strides3(const at::Tensor &t, int64_t *s)
{
    for (int i = 0; i < 3; ++i)
        s[i] = t.stride(i);
}

// Makes the tensors' device the current one and gives its current stream.
// (Host tensors have none: the library refuses their memory.)
struct Place {
    c10::OptionalDeviceGuard guard;
    void *stream = nullptr;
    explicit Place(const at::Tensor &t)
    {
        if (t.is_cuda()) {
            guard.reset_device(t.device());
            stream = c10::hip::getCurrentHIPStream(t.get_device()).stream();
        }
    }
};

at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, c10::Device d)
{
    const at::AutoDispatchBelowADInplaceOrView below;  // results are not recorded
    return at::empty(shape, at::TensorOptions().dtype(type).device(d));
}

struct Cache {
    seq_cache_t c;
    c10::Device device = c10::kCPU;
    at::ScalarType type;
};

// Memory that a call writes, asked for before that which it reads: a lazy copy gets
// its own first, and what shares its storage moves with it.
void *written(const at::Tensor &t) { return t.mutable_data_ptr(); }

// write: the call writes the pages and scales.
Cache cache(PyObject *k_pages, PyObject *v_pages, PyObject *table_, PyObject *k_scale, PyObject *v_scale, bool write)
{
    const auto memory = [write](const at::Tensor &t) { return write ? written(t) : const_cast<void *>(t.const_data_ptr()); };
    const at::Tensor &k = tensor(k_pages, "k_pages"), &v = tensor(v_pages, "v_pages"), &table = tensor(table_, "table");
    Cache r;
    r.device = k.device(), r.type = k.scalar_type();
    if (k.dim() != 4 || v.sizes() != k.sizes() || v.scalar_type() != r.type)
        refuse(PyExc_ValueError, "k_pages and v_pages must have one shape [pages][page][Hkv][D] and one type");
    dense_channels(k, "k_pages");
    dense_channels(v, "v_pages");
    if (table.dim() != 2 || table.scalar_type() != at::kInt || (table.size(1) > 1 && table.stride(1) != 1))
        refuse(PyExc_ValueError, "table must be an int32 [B][max_pages] tensor, dense in its last dimension");
    on_device(v, r.device);
    on_device(table, r.device);
    seq_cache_t &c = r.c;
    c.dt = code(r.type);
    c.pages = k.size(0), c.page = k.size(1), c.Hkv = k.size(2), c.D = k.size(3);
    c.B = table.size(0), c.max_pages = table.size(1);
    c.table_stride = c.B > 1 ? table.stride(0) : c.max_pages;
    strides3(k, c.k_stride);
    strides3(v, c.v_stride);
    c.k = memory(k), c.v = memory(v);
    c.table = (const int32_t *)table.const_data_ptr();
    c.k_scale = c.v_scale = nullptr;
    for (int i = 0; i < 3; ++i)
        c.k_scale_stride[i] = c.v_scale_stride[i] = 0;
    if (!coded(c.dt)) {
        if (k_scale != Py_None || v_scale != Py_None)
            refuse(PyExc_ValueError, "k_scale and v_scale go with 8-bit pages");
        return r;
    }
    if (k_scale == Py_None || v_scale == Py_None)
        refuse(PyExc_ValueError, "8-bit pages need k_scale and v_scale");
    const at::Tensor &ks = tensor(k_scale, "k_scale"), &vs = tensor(v_scale, "v_scale");
    const at::IntArrayRef shape = k.sizes().slice(0, 3);
    if (ks.sizes() != shape || vs.sizes() != shape || ks.scalar_type() != at::kFloat || vs.scalar_type() != at::kFloat)
        refuse(PyExc_ValueError, "k_scale and v_scale must be fp32 [pages][page][Hkv]");
    on_device(ks, r.device);
    on_device(vs, r.device);
    strides3(ks, c.k_scale_stride);
    strides3(vs, c.v_scale_stride);
    c.k_scale = (float *)memory(ks), c.v_scale = (float *)memory(vs);
    return r;
}

// k and v [B][L][Hkv][D] of a copy.
void dense(const Cache &c, const at::Tensor &k, const at::Tensor &v, int64_t L)
{
    if (k.dim() != 4 || k.size(0) != c.c.B || k.size(1) != L || k.size(2) != c.c.Hkv || k.size(3) != c.c.D ||
        v.sizes() != k.sizes())
        refuse(PyExc_ValueError, "k and v must be [B][L][Hkv][D], as the table and the pages have it");
    if (v.scalar_type() != k.scalar_type())
        refuse(PyExc_TypeError, "k and v must have one type");
    dense_channels(k, "k");
    dense_channels(v, "v");
    on_device(k, c.device);
    on_device(v, c.device);
}

int wide_type(const Cache &c, at::ScalarType t, const char *what)
{
    const int dt = code(t);
    if (coded(dt) || (!coded(c.c.dt) && dt != c.c.dt))
        refuse(PyExc_TypeError, "%s must have the type of the pages, or a wider one than 8-bit pages", what);
    return dt;
}

template <class F>
int64_t without_gil(F f)
{
    PyThreadState *const s = PyEval_SaveThread();
    const int64_t rc = f();
    PyEval_RestoreThread(s);
    return rc;
}

void expect(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want)
        refuse(PyExc_TypeError, "%zd arguments expected, %zd given", want, n);
}

// ---- the calls; seq_cache.py documents their arguments ----

// rotary(x, freq, positions, interleaved, amplitude, out, backward)
PyObject *rotary(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 7);
    const at::Tensor &x = tensor(args[0], "x"), &freq = tensor(args[1], "freq");
    if (x.dim() != 4)
        refuse(PyExc_ValueError, "x must have four dimensions");
    dense_channels(x, "x");
    if (freq.dim() != 1 || freq.scalar_type() != at::kDouble || !freq.is_cpu() || !freq.is_contiguous())
        refuse(PyExc_ValueError, "freq must be a contiguous fp64 [rot/2] tensor in host memory");
    seq_rotary_t a;
    a.dt = code(x.scalar_type()), a.interleaved = truth(args[3]), a.amplitude = (float)number(args[4]);
    a.B = x.size(0), a.L = x.size(1), a.H = x.size(2), a.D = x.size(3), a.rot = 2 * freq.size(0);
    a.by_token = 0, a.positions = nullptr;
    if (args[2] != Py_None) {
        const at::Tensor &p = tensor(args[2], "positions");
        a.by_token = p.dim() == 2;
        if (p.scalar_type() != at::kInt || p.dim() < 1 || p.dim() > 2 || p.size(0) != a.B ||
            (a.by_token && p.size(1) != a.L) || !p.is_contiguous())
            refuse(PyExc_ValueError, "positions must be a contiguous int32 [B] or [B][L] tensor");
        on_device(p, x.device());
        a.positions = (const int32_t *)p.const_data_ptr();
    }
    const bool backward = truth(args[6]);
    const Place place(x);
    at::Tensor out;
    if (args[5] == Py_None) {
        out = empty(x.sizes(), x.scalar_type(), x.device());
    } else {
        out = tensor(args[5], "out");
        like(out, x, "out");
    }
    strides3(x, a.x_stride);
    strides3(out, a.y_stride);
    a.freq = (const double *)freq.const_data_ptr();
    void *const to = written(out);
    const void *const from = x.const_data_ptr();
    check(without_gil([&] { return (backward ? seq_rotary_backward : seq_rotary_forward)(&a, from, to, place.stream); }),
          backward ? "seq_rotary_backward" : "seq_rotary_forward");
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// cache_write(k, v, k_pages, v_pages, table, start, count, k_scale, v_scale)
PyObject *cache_write(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 9);
    const Cache c = cache(args[2], args[3], args[4], args[7], args[8], true);
    const at::Tensor &k = tensor(args[0], "k"), &v = tensor(args[1], "v");
    const int64_t L = k.dim() == 4 ? k.size(1) : 0;
    dense(c, k, v, L);
    const int dt = wide_type(c, k.scalar_type(), "k and v");
    const int32_t *const start = counts(args[5], "start", c.c.B, c.device), *const count = counts(args[6], "count", c.c.B, c.device);
    int64_t ks[3], vs[3];
    strides3(k, ks);
    strides3(v, vs);
    const Place place(k);
    const void *const kp = k.const_data_ptr(), *const vp = v.const_data_ptr();
    check(without_gil([&] {
              return seq_cache_write(&c.c, kp, vp, ks, vs, L, (im2win_dtype_t)dt, start, count, place.stream);
          }),
          "seq_cache_write");
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// cache_read(k_pages, v_pages, table, length, L, dtype, k_scale, v_scale, k, v)
PyObject *cache_read(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 10);
    const Cache c = cache(args[0], args[1], args[2], args[6], args[7], false);
    const int64_t L = PyLong_AsLongLong(args[4]);
    if (L == -1 && PyErr_Occurred())
        throw python_error();
    if (L < 0)
        refuse(PyExc_ValueError, "L must not be negative");
    at::ScalarType type = coded(c.c.dt) ? at::kFloat : c.type;
    if (args[5] != Py_None) {
        if (!THPDtype_Check(args[5]))
            refuse(PyExc_TypeError, "dtype must be a torch type");
        type = ((THPDtype *)args[5])->scalar_type;
    }
    const int dt = wide_type(c, type, "the result");
    const int32_t *const len = counts(args[3], "length", c.c.B, c.device);
    if (!len && c.c.B > 0)
        refuse(PyExc_ValueError, "length must be a contiguous int32 [%lld] tensor", (long long)c.c.B);
    const Place place(tensor(args[0], "k_pages"));
    const int64_t shape[4] = {c.c.B, L, c.c.Hkv, c.c.D};
    at::Tensor out[2];
    for (int i = 0; i < 2; ++i) {
        if (args[8 + i] == Py_None) {
            out[i] = empty(shape, type, c.device);
        } else {
            out[i] = tensor(args[8 + i], i ? "v" : "k");
            if (out[i].scalar_type() != type)
                refuse(PyExc_ValueError, "k and v must have the type of the result");
        }
    }
    dense(c, out[0], out[1], L);
    int64_t ks[3], vs[3];
    strides3(out[0], ks);
    strides3(out[1], vs);
    void *const kp = written(out[0]), *const vp = written(out[1]);
    check(without_gil([&] { return seq_cache_read(&c.c, kp, vp, ks, vs, L, (im2win_dtype_t)dt, len, place.stream); }),
          "seq_cache_read");
    PyObject *const pair = PyTuple_New(2);
    if (!pair)
        throw python_error();
    for (int i = 0; i < 2; ++i)
        PyTuple_SET_ITEM(pair, i, THPVariable_Wrap(std::move(out[i])));
    return pair;
    END_HANDLE_TH_ERRORS
}

// paged_workspace_bytes(q, k_pages, v_pages, table, k_scale, v_scale)
PyObject *paged_workspace_bytes(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 6);
    const Cache c = cache(args[1], args[2], args[3], args[4], args[5], false);
    const at::Tensor &q = tensor(args[0], "q");
    if (q.dim() != 3)
        refuse(PyExc_ValueError, "q must be [B][H][D], as the table and the pages have it");
    const int64_t need = seq_paged_attention_workspace_bytes(&c.c, q.size(1), (im2win_dtype_t)code(q.scalar_type()));
    check(need, "seq_paged_attention_workspace_bytes");
    return PyLong_FromLongLong(need);
    END_HANDLE_TH_ERRORS
}

// paged_attention(q, k_pages, v_pages, table, length, scale, cap, bias, k_scale, v_scale, out, ws)
PyObject *paged_attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 12);
    const Cache c = cache(args[1], args[2], args[3], args[8], args[9], false);
    const at::Tensor &q = tensor(args[0], "q");
    if (q.dim() != 3 || q.size(0) != c.c.B || q.size(2) != c.c.D)
        refuse(PyExc_ValueError, "q must be [B][H][D], as the table and the pages have it");
    dense_channels(q, "q");
    on_device(q, c.device);
    seq_paged_attention_t a;
    a.dt = wide_type(c, q.scalar_type(), "q");
    a.H = q.size(1);
    a.scale = args[5] == Py_None ? (float)pow((double)c.c.D, -0.5) : (float)number(args[5]);
    a.cap = (float)number(args[6]);
    a.len = counts(args[4], "length", c.c.B, c.device);
    if (!a.len && c.c.B > 0)
        refuse(PyExc_ValueError, "length must be a contiguous int32 [%lld] tensor", (long long)c.c.B);
    a.R = 0, a.strip = nullptr;
    if (args[7] != Py_None) {
        const at::Tensor &bias = tensor(args[7], "bias");
        if (bias.dim() != 2 || bias.size(0) != a.H || bias.size(1) % 2 == 0 || bias.size(1) < 3 ||
            bias.scalar_type() != at::kFloat || !bias.is_contiguous())
            refuse(PyExc_ValueError, "bias must be a contiguous fp32 [H][2R+1] strip");
        on_device(bias, c.device);
        a.R = bias.size(1) / 2, a.strip = (const float *)bias.const_data_ptr();
    }
    const Place place(q);
    at::Tensor out, ws;
    if (args[10] == Py_None) {
        out = empty(q.sizes(), q.scalar_type(), c.device);
    } else {
        out = tensor(args[10], "out");
        like(out, q, "out");
    }
    at::Tensor lse = empty({c.c.B, a.H}, at::kFloat, c.device);
    if (args[11] != Py_None) {
        ws = tensor(args[11], "ws");
        if (!ws.is_contiguous())  // its bytes are numbered from the first
            refuse(PyExc_ValueError, "ws must be contiguous");
        on_device(ws, c.device);
    } else {
        const int64_t need = seq_paged_attention_workspace_bytes(&c.c, a.H, (im2win_dtype_t)a.dt);
        check(need, "seq_paged_attention_workspace_bytes");
        if (need)
            ws = empty({need}, at::kByte, c.device);
    }
    a.q_stride[0] = q.stride(0), a.q_stride[1] = q.stride(1);
    a.out_stride[0] = out.stride(0), a.out_stride[1] = out.stride(1);
    void *const op = written(out);
    float *const lp = (float *)written(lse);
    void *const wp = ws.defined() ? written(ws) : nullptr;
    const void *const qp = q.const_data_ptr();
    const int64_t size = ws.defined() ? (int64_t)ws.nbytes() : 0;
    check(without_gil([&] { return seq_paged_attention_forward(&c.c, &a, qp, op, lp, wp, size, place.stream); }),
          "seq_paged_attention_forward");
    PyObject *const pair = PyTuple_New(2);
    if (!pair)
        throw python_error();
    PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(std::move(out)));
    PyTuple_SET_ITEM(pair, 1, THPVariable_Wrap(std::move(lse)));
    return pair;
    END_HANDLE_TH_ERRORS
}

PyObject *set_error(PyObject *, PyObject *type)
{
    Py_INCREF(type);
    Py_XSETREF(g_error, type);
    Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"rotary", (PyCFunction)(void (*)(void))rotary, METH_FASTCALL, nullptr},
    {"cache_write", (PyCFunction)(void (*)(void))cache_write, METH_FASTCALL, nullptr},
    {"cache_read", (PyCFunction)(void (*)(void))cache_read, METH_FASTCALL, nullptr},
    {"paged_workspace_bytes", (PyCFunction)(void (*)(void))paged_workspace_bytes, METH_FASTCALL, nullptr},
    {"paged_attention", (PyCFunction)(void (*)(void))paged_attention, METH_FASTCALL, nullptr},
    {"set_error", set_error, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_seq_cache", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__seq_cache(void) { return PyModule_Create(&kModule); }

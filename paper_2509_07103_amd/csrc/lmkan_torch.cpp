// The per-call part of binding.py in native code: check the tensors, allocate what the caller did not
// bring, find the current stream, call the library.  With tables and batches small enough for one
// launch per call, marshalling in Python took longer than the GPU did (forward 12.4 us per call, of
// which the library and its launch are 4).
//
// Only the ordinary case is handled here.  Anything else (a tensor of the wrong type, shape or device, a
// status other than LMKAN_OK) makes a function return None without having launched anything that
// counts, and binding.py goes its own way, which raises the error that describes it.
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>

#include "lmkan.h"

namespace {

// addresses of the library that binding.py has loaded
struct Library {
    decltype(&lmkan_workspace_bytes) workspace_bytes;
    decltype(&lmkan_packed_bytes) packed_bytes;
    decltype(&lmkan_forward) forward;
    decltype(&lmkan_backward) backward;
    decltype(&lmkan_conv2d_rows) conv2d_rows;
    decltype(&lmkan_conv2d_forward) conv2d_forward;
    decltype(&lmkan_conv2d_backward) conv2d_backward;
    decltype(&lmkan_pack) pack;
    decltype(&lmkan_orthogonalize_workspace_bytes) orthogonalize_workspace_bytes;
    decltype(&lmkan_orthogonalize) orthogonalize;
    decltype(&lmkan_muon_step) muon_step;
    decltype(&lmkan_linear_i8_workspace_bytes) linear_i8_workspace_bytes;
    decltype(&lmkan_linear_i8) linear_i8;
    decltype(&lmkan_checkpoint_rows) checkpoint_rows;
    decltype(&lmkan_restore_rows) restore_rows;
    decltype(&lmkan_layer_norm) layer_norm;
    decltype(&lmkan_layer_norm_backward_workspace_bytes) layer_norm_backward_workspace_bytes;
    decltype(&lmkan_layer_norm_backward) layer_norm_backward;
    decltype(&lmkan_linear_grad_workspace_bytes) linear_grad_workspace_bytes;
    decltype(&lmkan_linear_grad) linear_grad;
    decltype(&lmkan_adapters_workspace_bytes) adapters_workspace_bytes;
    decltype(&lmkan_adapters_add) adapters_add;
} g_lib;

// attribute names, interned once
enum { kNIn, kNOut, kGrid, kOrder, kDtype, kLayout, kFlags, kDescNames };
enum { kN, kH, kW, kCIn, kKh, kKw, kStride, kConvNames };
enum { kBatch, kRows, kCols, kMatrixDtype, kMatrixNames };
enum { kLinIn, kLinOut, kXDtype, kYDtype, kRelu, kLinearNames };
PyObject *g_desc_names[kDescNames], *g_conv_names[kConvNames], *g_matrix_names[kMatrixNames], *g_linear_names[kLinearNames], *g_eps_name;
enum { kLr, kMomentum, kDecay, kScale, kNesterov, kMuonNames };
PyObject *g_muon_names[kMuonNames];
enum { kNormCols, kNormX, kNormY, kNormNames };
enum { kCount, kRank, kAdapterIn, kAdapterOut, kAdapterDtype, kAdapterX, kAdapterY, kAdapterRelu, kAdapterNames };
PyObject *g_norm_names[kNormNames], *g_adapter_names[kAdapterNames];

template <int N>
bool read_ints(PyObject *obj, PyObject *const (&names)[N], int32_t (&out)[N])
{
    for (int i = 0; i < N; ++i) {
        PyObject *v = PyObject_GetAttr(obj, names[i]);
        const long n = v ? PyLong_AsLong(v) : -1;
        Py_XDECREF(v);
        if ((n == -1 && PyErr_Occurred()) || n < INT32_MIN || n > INT32_MAX) {
            PyErr_Clear();
            return false;
        }
        out[i] = (int32_t)n;
    }
    return true;
}

bool read_desc(PyObject *obj, lmkan_desc &d)
{
    int32_t v[kDescNames];
    if (!read_ints(obj, g_desc_names, v)) return false;
    d = {v[kNIn], v[kNOut], v[kGrid], v[kOrder], v[kDtype], v[kLayout], v[kFlags]};
    return d.n_in >= 2 && d.n_out >= 1 && d.grid >= 3 && d.grid <= LMKAN_MAX_GRID && d.coef_dtype >= 0 && d.coef_dtype <= 2;
}

bool read_double(PyObject *obj, PyObject *name, double &out)
{
    PyObject *v = PyObject_GetAttr(obj, name);
    out = v ? PyFloat_AsDouble(v) : -1.0;
    Py_XDECREF(v);
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}

at::ScalarType type_of(int dtype) { return dtype == LMKAN_F32 ? at::kFloat : dtype == LMKAN_F16 ? at::kHalf : at::kBFloat16; }
bool known_dtype(int dtype) { return dtype == LMKAN_F32 || dtype == LMKAN_F16 || dtype == LMKAN_BF16; }

at::ScalarType coef_type(const lmkan_desc &d) { return type_of(d.coef_dtype); }

// the tensor behind a Python object, or nullptr
const at::Tensor *tensor(PyObject *o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

bool fits(const at::Tensor *t, at::ScalarType type, at::IntArrayRef shape)
{
    return t && t->is_cuda() && t->scalar_type() == type && t->sizes() == shape && t->is_contiguous();
}

std::array<int64_t, 4> coef_shape(const lmkan_desc &d) { return {d.grid + 1, d.grid + 1, d.n_in / 2, d.n_out}; }

bool coef_fits(const lmkan_desc &d, const at::Tensor *t)
{
    if (d.coef_layout == LMKAN_LAYOUT_PACKED)
        return fits(t, coef_type(d), {(int64_t)(g_lib.packed_bytes(&d) / (d.coef_dtype == LMKAN_F32 ? 4 : 2))});
    return fits(t, coef_type(d), coef_shape(d));
}

void *data(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

void *current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// the caller's workspace, or one of the size the library asks for
bool workspace(PyObject *given, const lmkan_desc &d, int64_t rows, int pass, const at::Tensor &like, at::Tensor &ws, size_t &bytes)
{
    if (given != Py_None) {
        const at::Tensor *t = tensor(given);
        if (!t || !t->is_cuda() || !t->is_contiguous()) return false;
        ws = *t;
        bytes = t->nbytes();
        return true;
    }
    bytes = g_lib.workspace_bytes(&d, rows, pass);
    if (bytes > 0) ws = at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
    return true;
}

// an output the caller brought, or a new one
bool output(PyObject *given, at::IntArrayRef shape, const at::Tensor &like, at::Tensor &out)
{
    if (given == Py_None) {
        out = at::empty(shape, like.options());
        return true;
    }
    const at::Tensor *t = tensor(given);
    if (!fits(t, at::kFloat, shape)) return false;
    out = *t;
    return true;
}

PyObject *wrap(const at::Tensor &t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}

// geometry of a convolution (conv not None): shapes of the image and of the output, rows of the layer
struct Rows {
    lmkan_conv2d conv;
    bool is_conv = false;
    int64_t rows = 0;
    std::vector<int64_t> in, out;
};

bool read_rows(PyObject *conv, const lmkan_desc &d, const at::Tensor *x, Rows &r)
{
    if (!x) return false;
    if (conv == Py_None) {
        if (x->dim() != 2) return false;
        r.rows = x->size(0);
        r.in = {r.rows, d.n_in};
        r.out = {r.rows, d.n_out};
    } else {
        int32_t v[kConvNames], oh = 0, ow = 0;
        if (!read_ints(conv, g_conv_names, v)) return false;
        r.conv = {v[kN], v[kH], v[kW], v[kCIn], v[kKh], v[kKw], v[kStride]};
        r.is_conv = true;
        r.rows = g_lib.conv2d_rows(&r.conv, &oh, &ow);
        r.in = {v[kN], v[kH], v[kW], v[kCIn]};
        r.out = {v[kN], oh, ow, d.n_out};
    }
    return r.rows >= 0 && fits(x, at::kFloat, r.in);
}

// The Python exception of a C++ one, as torch's own functions raise it: running out of memory stays
// torch.OutOfMemoryError, which callers catch to go on with a smaller batch
PyObject *raise_in_python(const std::exception_ptr &e)
{
    torch::translate_exception_to_python(e);
    return nullptr;
}

// every function: arguments by position, None when binding.py has to take over
#define LMKAN_GUARDED_BEGIN try {
#define LMKAN_GUARDED_END                                                  \
    }                                                                      \
    catch (...)                                                            \
    {                                                                      \
        return raise_in_python(std::current_exception());                  \
    }

// forward(desc, conv, x, coef, y, workspace) -> y
PyObject *forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    lmkan_desc d;
    Rows r;
    const at::Tensor *x = tensor(args[2]), *coef = tensor(args[3]);
    at::Tensor y, ws;
    size_t bytes = 0;
    if (!read_desc(args[0], d) || !read_rows(args[1], d, x, r) || !coef_fits(d, coef) ||
        !output(args[4], r.out, *x, y) || !workspace(args[5], d, r.rows, 0, *x, ws, bytes))
        Py_RETURN_NONE;
    lmkan_status st;
    float *xp = static_cast<float *>(data(*x)), *yp = static_cast<float *>(data(y));
    void *s = current_stream(), *cp = data(*coef), *wp = data(ws);
    Py_BEGIN_ALLOW_THREADS
    st = r.is_conv ? g_lib.conv2d_forward(&d, &r.conv, xp, cp, yp, wp, bytes, s)
                   : g_lib.forward(&d, r.rows, xp, cp, yp, wp, bytes, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    return wrap(y);
    LMKAN_GUARDED_END
}

// backward(desc, conv, x, coef, grad_y, need_x, need_coef, grad_x, grad_coef, workspace) -> (grad_x, grad_coef)
PyObject *backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 10) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    lmkan_desc d;
    Rows r;
    const at::Tensor *x = tensor(args[2]), *coef = tensor(args[3]), *gy = tensor(args[4]);
    const bool need_x = args[5] == Py_True, need_coef = args[6] == Py_True;
    if ((!need_x && args[5] != Py_False) || (!need_coef && args[6] != Py_False)) Py_RETURN_NONE;
    at::Tensor gx, gp, ws;
    size_t bytes = 0;
    if (!read_desc(args[0], d) || !read_rows(args[1], d, x, r) || !(args[3] == Py_None || coef_fits(d, coef)) ||
        !fits(gy, at::kFloat, r.out))
        Py_RETURN_NONE;
    if (need_coef && args[8] == Py_None && (d.flags & LMKAN_FLAG_ACCUMULATE_GRAD_COEF)) Py_RETURN_NONE;
    if ((need_x && !output(args[7], r.in, *x, gx)) || (need_coef && !output(args[8], coef_shape(d), *x, gp)) ||
        !workspace(args[9], d, r.rows, need_x && need_coef ? 1 : need_x ? 2 : 3, *x, ws, bytes))
        Py_RETURN_NONE;
    lmkan_status st;
    float *xp = static_cast<float *>(data(*x)), *gyp = static_cast<float *>(data(*gy));
    float *gxp = static_cast<float *>(data(gx)), *gpp = static_cast<float *>(data(gp));
    void *s = current_stream(), *cp = coef ? data(*coef) : nullptr, *wp = data(ws);
    Py_BEGIN_ALLOW_THREADS
    st = r.is_conv ? g_lib.conv2d_backward(&d, &r.conv, xp, cp, gyp, gxp, gpp, wp, bytes, s)
                   : g_lib.backward(&d, r.rows, xp, cp, gyp, gxp, gpp, wp, bytes, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    PyObject *a = wrap(gx), *b = wrap(gp), *pair = a && b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return pair;
    LMKAN_GUARDED_END
}

// pack(desc, coef) -> packed table
PyObject *pack(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 2) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    lmkan_desc d;
    const at::Tensor *coef = tensor(args[1]);
    if (!read_desc(args[0], d) || !fits(coef, coef_type(d), coef_shape(d))) Py_RETURN_NONE;
    const int64_t elems = (int64_t)(g_lib.packed_bytes(&d) / (d.coef_dtype == LMKAN_F32 ? 4 : 2));
    if (elems == 0) Py_RETURN_NONE;
    const at::Tensor out = at::empty({elems}, coef->options());
    lmkan_status st;
    void *s = current_stream(), *src = data(*coef), *dst = data(out);
    Py_BEGIN_ALLOW_THREADS
    st = g_lib.pack(&d, src, dst, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    return wrap(out);
    LMKAN_GUARDED_END
}

// a batch of matrices, and the (a, b, c) of a schedule's steps as the binding keeps them: bytes of float32
struct Matrices {
    lmkan_matrices d;
    const float *schedule;
    int32_t steps;
};

bool read_matrices(PyObject *desc, PyObject *schedule, Matrices &m)
{
    int32_t v[kMatrixNames];
    double eps;
    if (!read_ints(desc, g_matrix_names, v) || !read_double(desc, g_eps_name, eps) || !PyBytes_Check(schedule)) return false;
    m.d = {v[kBatch], v[kRows], v[kCols], v[kMatrixDtype], (float)eps};
    m.steps = (int32_t)(PyBytes_GET_SIZE(schedule) / (3 * sizeof(float)));
    m.schedule = reinterpret_cast<const float *>(PyBytes_AS_STRING(schedule));
    return m.d.batch >= 0 && m.d.rows >= 1 && m.d.cols >= 1 && known_dtype(m.d.dtype);
}

bool any_workspace(PyObject *given, size_t need, const at::Tensor &like, at::Tensor &ws, size_t &bytes)
{
    if (given != Py_None) {
        const at::Tensor *t = tensor(given);
        if (!t || !t->is_cuda() || !t->is_contiguous()) return false;
        ws = *t;
        bytes = t->nbytes();
        return true;
    }
    bytes = need;
    if (bytes > 0) ws = at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
    return true;
}

// orthogonalize(desc, schedule, x, out, workspace) -> out
PyObject *orthogonalize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 5) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    Matrices m;
    if (!read_matrices(args[0], args[1], m)) Py_RETURN_NONE;
    const at::ScalarType type = type_of(m.d.dtype);
    const std::array<int64_t, 3> shape = {m.d.batch, m.d.rows, m.d.cols};
    const at::Tensor *x = tensor(args[2]);
    if (!fits(x, type, shape)) Py_RETURN_NONE;
    at::Tensor out, ws;
    size_t bytes = 0;
    if (args[3] != Py_None) {
        const at::Tensor *t = tensor(args[3]);
        if (!fits(t, type, shape)) Py_RETURN_NONE;
        out = *t;
    } else {
        out = at::empty(shape, x->options());
    }
    if (!any_workspace(args[4], g_lib.orthogonalize_workspace_bytes(&m.d), *x, ws, bytes)) Py_RETURN_NONE;
    lmkan_status st;
    void *s = current_stream(), *xp = data(*x), *op = data(out), *wp = data(ws);
    Py_BEGIN_ALLOW_THREADS
    st = g_lib.orthogonalize(&m.d, m.steps, m.schedule, xp, op, wp, bytes, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    return wrap(out);
    LMKAN_GUARDED_END
}

// muon_step(desc, muon, schedule, grad, momentum, weight, workspace) -> weight
PyObject *muon_step(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 7) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    Matrices m;
    double p[kMuonNames];
    if (!read_matrices(args[0], args[2], m)) Py_RETURN_NONE;
    for (int i = 0; i < kMuonNames; ++i)
        if (!read_double(args[1], g_muon_names[i], p[i])) Py_RETURN_NONE;
    const lmkan_muon muon = {(float)p[kLr], (float)p[kMomentum], (float)p[kDecay], (float)p[kScale], p[kNesterov] != 0.0};
    const std::array<int64_t, 3> shape = {m.d.batch, m.d.rows, m.d.cols};
    const at::Tensor *grad = tensor(args[3]), *momentum = tensor(args[4]), *weight = tensor(args[5]);
    if (!fits(grad, type_of(m.d.dtype), shape) || !fits(momentum, at::kFloat, shape) || !fits(weight, at::kFloat, shape)) Py_RETURN_NONE;
    at::Tensor ws;
    size_t bytes = 0;
    if (!any_workspace(args[6], g_lib.orthogonalize_workspace_bytes(&m.d), *grad, ws, bytes)) Py_RETURN_NONE;
    lmkan_status st;
    float *mp = static_cast<float *>(data(*momentum)), *wp = static_cast<float *>(data(*weight));
    void *s = current_stream(), *gp = data(*grad), *sp = data(ws);
    Py_BEGIN_ALLOW_THREADS
    st = g_lib.muon_step(&m.d, &muon, m.steps, m.schedule, gp, mp, wp, sp, bytes, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    Py_INCREF(args[5]);
    return args[5];
    LMKAN_GUARDED_END
}

// linear_i8(desc, x, w_codes, w_scale, bias, beta, y, workspace) -> y
PyObject *linear_i8(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 8) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    int32_t v[kLinearNames];
    if (!read_ints(args[0], g_linear_names, v) || !known_dtype(v[kXDtype]) || !known_dtype(v[kYDtype])) Py_RETURN_NONE;
    const lmkan_linear d = {v[kLinIn], v[kLinOut], v[kXDtype], v[kYDtype], v[kRelu] ? LMKAN_LINEAR_RELU : 0};
    const at::Tensor *x = tensor(args[1]), *w = tensor(args[2]), *scale = tensor(args[3]), *bias = tensor(args[4]);
    const double beta = PyFloat_AsDouble(args[5]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (!x || x->dim() != 2) Py_RETURN_NONE;
    const int64_t batch = x->size(0);
    if (!fits(x, type_of(d.x_dtype), {batch, d.n_in}) || !fits(w, at::kChar, {d.n_out, d.n_in}) || !fits(scale, at::kFloat, {d.n_out}) ||
        !(args[4] == Py_None || fits(bias, at::kFloat, {d.n_out})))
        Py_RETURN_NONE;
    at::Tensor y, ws;
    size_t bytes = 0;
    if (args[6] != Py_None) {
        const at::Tensor *t = tensor(args[6]);
        if (!fits(t, type_of(d.y_dtype), {batch, d.n_out})) Py_RETURN_NONE;
        y = *t;
    } else {
        if (beta != 0.0) Py_RETURN_NONE;
        y = at::empty({batch, d.n_out}, x->options().dtype(type_of(d.y_dtype)));
    }
    if (!any_workspace(args[7], g_lib.linear_i8_workspace_bytes(&d, batch), *x, ws, bytes)) Py_RETURN_NONE;
    lmkan_status st;
    const int8_t *cp = static_cast<const int8_t *>(data(*w));
    const float *sp = static_cast<const float *>(data(*scale)), *bp = bias ? static_cast<const float *>(data(*bias)) : nullptr;
    void *s = current_stream(), *xp = data(*x), *yp = data(y), *wp = data(ws);
    Py_BEGIN_ALLOW_THREADS
    st = g_lib.linear_i8(&d, batch, xp, cp, sp, bp, (float)beta, yp, wp, bytes, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    return wrap(y);
    LMKAN_GUARDED_END
}

// The operators on rows.  Tensors are on the current device, where the library launches; every output that the caller
// did not bring is allocated like `like`.
bool here(const at::Tensor *t, at::ScalarType type, at::IntArrayRef shape)
{
    return fits(t, type, shape) && t->device().index() == c10::hip::current_device();
}
bool here_or_none(PyObject *o, at::ScalarType type, at::IntArrayRef shape) { return o == Py_None || here(tensor(o), type, shape); }

bool made(PyObject *given, at::ScalarType type, at::IntArrayRef shape, const at::Tensor &like, at::Tensor &out)
{
    if (given == Py_None) {
        out = at::empty(shape, like.options().dtype(type));
        return true;
    }
    const at::Tensor *t = tensor(given);
    if (!here(t, type, shape)) return false;
    out = *t;
    return true;
}

bool workspace_here(PyObject *given, size_t need, const at::Tensor &like, at::Tensor &ws, size_t &bytes)
{
    return any_workspace(given, need, like, ws, bytes) && (given == Py_None || ws.device().index() == c10::hip::current_device());
}

template <class T>
T *data_or_null(PyObject *o)
{
    const at::Tensor *t = o == Py_None ? nullptr : tensor(o);
    return t ? static_cast<T *>(t->data_ptr()) : nullptr;
}

bool truth(PyObject *o, bool &v)
{
    v = o == Py_True;
    return v || o == Py_False;
}

int64_t exps_of(int64_t cols) { return (cols + LMKAN_CHECKPOINT_BLOCK - 1) / LMKAN_CHECKPOINT_BLOCK; }

// a tuple of objects, which it takes
template <class... P>
PyObject *tuple_of(P... objects)
{
    PyObject *all[] = {objects...};
    bool whole = true;
    for (PyObject *o : all) whole = whole && o;
    PyObject *t = whole ? PyTuple_Pack((Py_ssize_t)sizeof...(P), objects...) : nullptr;
    for (PyObject *o : all) Py_XDECREF(o);
    return t;
}

// checkpoint_rows(x, relu) -> (codes, exps)
PyObject *checkpoint_rows(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 2) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    const at::Tensor *x = tensor(args[0]);
    bool relu;
    if (!x || x->dim() != 2 || !truth(args[1], relu)) Py_RETURN_NONE;
    const int dtype = x->scalar_type() == at::kFloat ? LMKAN_F32 : x->scalar_type() == at::kHalf ? LMKAN_F16 : LMKAN_BF16;
    const int64_t rows = x->size(0), cols = x->size(1);
    if (!here(x, type_of(dtype), {rows, cols}) || cols > LMKAN_MAX_N_IN) Py_RETURN_NONE;
    const at::Tensor codes = at::empty({rows, cols}, x->options().dtype(at::kChar)), exps = at::empty({rows, exps_of(cols)}, x->options().dtype(at::kByte));
    lmkan_status st;
    void *s = current_stream(), *xp = data(*x);
    int8_t *cp = static_cast<int8_t *>(data(codes));
    uint8_t *ep = static_cast<uint8_t *>(data(exps));
    Py_BEGIN_ALLOW_THREADS
    st = g_lib.checkpoint_rows(rows, (int32_t)cols, dtype, relu ? LMKAN_LINEAR_RELU : 0, xp, cp, ep, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    return tuple_of(wrap(codes), wrap(exps));
    LMKAN_GUARDED_END
}

// restore_rows(codes, exps, weight, bias, relu, dtype, y) -> y
PyObject *restore_rows(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 7) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    const at::Tensor *codes = tensor(args[0]), *exps = tensor(args[1]);
    bool relu;
    if (!codes || codes->dim() != 2 || !truth(args[4], relu) || !PyLong_Check(args[5])) Py_RETURN_NONE;
    const long dtype = PyLong_AsLong(args[5]);
    if (dtype == -1 && PyErr_Occurred()) PyErr_Clear();
    const int64_t rows = codes->size(0), cols = codes->size(1);
    if (dtype < 0 || dtype > 2 || cols > LMKAN_MAX_N_IN || !here(codes, at::kChar, {rows, cols}) || !here(exps, at::kByte, {rows, exps_of(cols)}) ||
        !here_or_none(args[2], at::kFloat, {cols}) || !here_or_none(args[3], at::kFloat, {cols}))
        Py_RETURN_NONE;
    at::Tensor y;
    if (!made(args[6], type_of((int)dtype), {rows, cols}, *codes, y)) Py_RETURN_NONE;
    lmkan_status st;
    void *s = current_stream(), *yp = data(y);
    const int8_t *cp = static_cast<int8_t *>(data(*codes));
    const uint8_t *ep = static_cast<uint8_t *>(data(*exps));
    const float *wp = data_or_null<float>(args[2]), *bp = data_or_null<float>(args[3]);
    Py_BEGIN_ALLOW_THREADS
    st = g_lib.restore_rows(rows, (int32_t)cols, (int32_t)dtype, relu ? LMKAN_LINEAR_RELU : 0, cp, ep, wp, bp, yp, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    return wrap(y);
    LMKAN_GUARDED_END
}

bool read_norm(PyObject *desc, bool accumulate, lmkan_norm &d)
{
    int32_t v[kNormNames];
    double eps;
    if (!read_ints(desc, g_norm_names, v) || !read_double(desc, g_eps_name, eps)) return false;
    d = {v[kNormCols], v[kNormX], v[kNormY], accumulate ? LMKAN_NORM_ACCUMULATE : 0, (float)eps};
    return d.cols >= 1 && d.cols <= LMKAN_MAX_N_IN && known_dtype(d.x_dtype) && known_dtype(d.y_dtype);
}

// layer_norm(desc, x, weight, bias, y, keep) -> (y, stats, (codes, exps) or None)
PyObject *layer_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    lmkan_norm d;
    bool keep;
    const at::Tensor *x = tensor(args[1]);
    if (!read_norm(args[0], false, d) || !truth(args[5], keep) || !x || x->dim() != 2) Py_RETURN_NONE;
    const int64_t rows = x->size(0);
    if (!here(x, type_of(d.x_dtype), {rows, d.cols}) || !here_or_none(args[2], at::kFloat, {d.cols}) || !here_or_none(args[3], at::kFloat, {d.cols}))
        Py_RETURN_NONE;
    at::Tensor y, codes, exps;
    if (!made(args[4], type_of(d.y_dtype), {rows, d.cols}, *x, y)) Py_RETURN_NONE;
    const at::Tensor stats = at::empty({rows, 2}, x->options().dtype(at::kFloat));
    if (keep) {
        codes = at::empty({rows, d.cols}, x->options().dtype(at::kChar));
        exps = at::empty({rows, exps_of(d.cols)}, x->options().dtype(at::kByte));
    }
    lmkan_status st;
    void *s = current_stream(), *xp = data(*x), *yp = data(y);
    const float *wp = data_or_null<float>(args[2]), *bp = data_or_null<float>(args[3]);
    float *sp = static_cast<float *>(data(stats));
    int8_t *cp = static_cast<int8_t *>(data(codes));
    uint8_t *ep = static_cast<uint8_t *>(data(exps));
    Py_BEGIN_ALLOW_THREADS
    st = g_lib.layer_norm(&d, rows, xp, wp, bp, yp, sp, cp, ep, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    PyObject *kept = Py_None;
    if (keep) kept = tuple_of(wrap(codes), wrap(exps));
    else Py_INCREF(kept);
    return tuple_of(wrap(y), wrap(stats), kept);
    LMKAN_GUARDED_END
}

// layer_norm_backward(desc, grad_y, stats, x, codes, exps, weight, need_x, need_weight, need_bias, grad_x, grad_weight,
//                     grad_bias, accumulate, workspace) -> (grad_x, grad_weight, grad_bias)
PyObject *layer_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 15) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    lmkan_norm d;
    bool need_x, need_weight, need_bias, accumulate;
    const at::Tensor *gy = tensor(args[1]), *stats = tensor(args[2]);
    if (!truth(args[7], need_x) || !truth(args[8], need_weight) || !truth(args[9], need_bias) || !truth(args[13], accumulate) ||
        !read_norm(args[0], accumulate, d) || !gy || gy->dim() != 2)
        Py_RETURN_NONE;
    const int64_t rows = gy->size(0);
    const at::ScalarType type = type_of(d.x_dtype);
    if (!here(gy, type_of(d.y_dtype), {rows, d.cols}) || !here(stats, at::kFloat, {rows, 2}) || !here_or_none(args[3], type, {rows, d.cols}) ||
        !here_or_none(args[4], at::kChar, {rows, d.cols}) || !here_or_none(args[5], at::kByte, {rows, exps_of(d.cols)}) ||
        !here_or_none(args[6], at::kFloat, {d.cols}))
        Py_RETURN_NONE;
    at::Tensor gx, gw, gb, ws;
    size_t bytes = 0;
    if ((need_x && !made(args[10], type, {rows, d.cols}, *gy, gx)) || (need_weight && !made(args[11], at::kFloat, {d.cols}, *gy, gw)) ||
        (need_bias && !made(args[12], at::kFloat, {d.cols}, *gy, gb)) ||
        !workspace_here(args[14], need_weight || need_bias ? g_lib.layer_norm_backward_workspace_bytes(&d, rows) : 0, *gy, ws, bytes))
        Py_RETURN_NONE;
    lmkan_status st;
    void *s = current_stream(), *gyp = data(*gy), *gxp = data(gx), *wsp = data(ws);
    const void *xp = data_or_null<void>(args[3]);
    const int8_t *cp = data_or_null<int8_t>(args[4]);
    const uint8_t *ep = data_or_null<uint8_t>(args[5]);
    const float *sp = static_cast<float *>(data(*stats)), *wp = data_or_null<float>(args[6]);
    float *gwp = static_cast<float *>(data(gw)), *gbp = static_cast<float *>(data(gb));
    Py_BEGIN_ALLOW_THREADS
    st = g_lib.layer_norm_backward(&d, rows, xp, cp, ep, sp, wp, gyp, gxp, gwp, gbp, wsp, bytes, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    return tuple_of(wrap(gx), wrap(gw), wrap(gb));
    LMKAN_GUARDED_END
}

// linear_grad(desc, codes, exps, grad_y, need_bias, grad_weight, grad_bias, accumulate, workspace) -> (grad_weight, grad_bias)
PyObject *linear_grad(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 9) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    int32_t v[kLinearNames];
    bool need_bias, accumulate;
    const at::Tensor *codes = tensor(args[1]), *exps = tensor(args[2]), *gy = tensor(args[3]);
    if (!read_ints(args[0], g_linear_names, v) || !known_dtype(v[kXDtype]) || !known_dtype(v[kYDtype]) || !truth(args[4], need_bias) ||
        !truth(args[7], accumulate) || !gy || gy->dim() != 2)
        Py_RETURN_NONE;
    const lmkan_linear d = {v[kLinIn], v[kLinOut], v[kXDtype], v[kYDtype], (v[kRelu] ? LMKAN_LINEAR_RELU : 0) | (accumulate ? LMKAN_LINEAR_ACCUMULATE : 0)};
    const int64_t batch = gy->size(0);
    if (d.n_in < 1 || d.n_out < 1 || !here(gy, type_of(d.y_dtype), {batch, d.n_out}) || !here(codes, at::kChar, {batch, d.n_in}) ||
        !here(exps, at::kByte, {batch, exps_of(d.n_in)}))
        Py_RETURN_NONE;
    at::Tensor gw, gb, ws;
    size_t bytes = 0;
    if (!made(args[5], at::kFloat, {d.n_out, d.n_in}, *gy, gw) || (need_bias && !made(args[6], at::kFloat, {d.n_out}, *gy, gb)) ||
        !workspace_here(args[8], g_lib.linear_grad_workspace_bytes(&d, batch), *gy, ws, bytes))
        Py_RETURN_NONE;
    lmkan_status st;
    void *s = current_stream(), *gyp = data(*gy), *wsp = data(ws);
    const int8_t *cp = static_cast<int8_t *>(data(*codes));
    const uint8_t *ep = static_cast<uint8_t *>(data(*exps));
    float *gwp = static_cast<float *>(data(gw)), *gbp = static_cast<float *>(data(gb));
    Py_BEGIN_ALLOW_THREADS
    st = g_lib.linear_grad(&d, batch, cp, ep, gyp, gwp, gbp, wsp, bytes, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    return tuple_of(wrap(gw), wrap(gb));
    LMKAN_GUARDED_END
}

// adapters_add(desc, x, index, a, b, y, scale, workspace) -> y
PyObject *adapters_add(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 8) Py_RETURN_NONE;
    LMKAN_GUARDED_BEGIN
    int32_t v[kAdapterNames];
    const at::Tensor *x = tensor(args[1]), *index = tensor(args[2]), *a = tensor(args[3]), *b = tensor(args[4]), *y = tensor(args[5]);
    if (!read_ints(args[0], g_adapter_names, v) || !known_dtype(v[kAdapterDtype]) || !known_dtype(v[kAdapterX]) || !known_dtype(v[kAdapterY]) || !x ||
        x->dim() != 2)
        Py_RETURN_NONE;
    const lmkan_adapters d = {v[kCount], v[kRank], v[kAdapterIn], v[kAdapterOut], v[kAdapterDtype], v[kAdapterX], v[kAdapterY],
                              v[kAdapterRelu] ? LMKAN_LINEAR_RELU : 0};
    const int64_t batch = x->size(0);
    const at::ScalarType type = type_of(d.dtype);
    if (!here(x, type_of(d.x_dtype), {batch, d.n_in}) || !here(index, at::kInt, {batch}) || !here(a, type, {d.count, d.rank, d.n_in}) ||
        !here(b, type, {d.count, d.n_out, d.rank}) || !here(y, type_of(d.y_dtype), {batch, d.n_out}) || !here_or_none(args[6], at::kFloat, {d.count}))
        Py_RETURN_NONE;
    at::Tensor ws;
    size_t bytes = 0;
    if (!workspace_here(args[7], g_lib.adapters_workspace_bytes(&d, batch), *x, ws, bytes)) Py_RETURN_NONE;
    lmkan_status st;
    void *s = current_stream(), *xp = data(*x), *ap = data(*a), *bp = data(*b), *yp = data(*y), *wsp = data(ws);
    const int32_t *ip = static_cast<int32_t *>(data(*index));
    const float *sp = data_or_null<float>(args[6]);
    Py_BEGIN_ALLOW_THREADS
    st = g_lib.adapters_add(&d, batch, xp, ip, ap, bp, sp, yp, wsp, bytes, s);
    Py_END_ALLOW_THREADS
    if (st != LMKAN_OK) Py_RETURN_NONE;
    Py_INCREF(args[5]);
    return args[5];
    LMKAN_GUARDED_END
}

// init(the addresses, in the order of Library)
PyObject *init(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != (Py_ssize_t)(sizeof(Library) / sizeof(void *))) {
        PyErr_SetString(PyExc_ValueError, "init: one address per library function");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < n; ++i) {
        void *p = PyLong_AsVoidPtr(args[i]);
        if (!p) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "init: null address");
            return nullptr;
        }
        reinterpret_cast<void **>(&g_lib)[i] = p;
    }
    Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {{"init", (PyCFunction)(void (*)(void))init, METH_FASTCALL, nullptr},
                           {"forward", (PyCFunction)(void (*)(void))forward, METH_FASTCALL, nullptr},
                           {"backward", (PyCFunction)(void (*)(void))backward, METH_FASTCALL, nullptr},
                           {"pack", (PyCFunction)(void (*)(void))pack, METH_FASTCALL, nullptr},
                           {"orthogonalize", (PyCFunction)(void (*)(void))orthogonalize, METH_FASTCALL, nullptr},
                           {"muon_step", (PyCFunction)(void (*)(void))muon_step, METH_FASTCALL, nullptr},
                           {"linear_i8", (PyCFunction)(void (*)(void))linear_i8, METH_FASTCALL, nullptr},
                           {"checkpoint_rows", (PyCFunction)(void (*)(void))checkpoint_rows, METH_FASTCALL, nullptr},
                           {"restore_rows", (PyCFunction)(void (*)(void))restore_rows, METH_FASTCALL, nullptr},
                           {"layer_norm", (PyCFunction)(void (*)(void))layer_norm, METH_FASTCALL, nullptr},
                           {"layer_norm_backward", (PyCFunction)(void (*)(void))layer_norm_backward, METH_FASTCALL, nullptr},
                           {"linear_grad", (PyCFunction)(void (*)(void))linear_grad, METH_FASTCALL, nullptr},
                           {"adapters_add", (PyCFunction)(void (*)(void))adapters_add, METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void)
{
    static const char *desc[] = {"n_in", "n_out", "grid", "spline_order", "coef_dtype", "coef_layout", "flags"};
    static const char *conv[] = {"n", "h", "w", "c_in", "kh", "kw", "stride"};
    for (int i = 0; i < kDescNames; ++i) g_desc_names[i] = PyUnicode_InternFromString(desc[i]);
    for (int i = 0; i < kConvNames; ++i) g_conv_names[i] = PyUnicode_InternFromString(conv[i]);
    static const char *matrix[] = {"batch", "rows", "cols", "dtype"};
    static const char *muon[] = {"lr", "momentum", "weight_decay", "scale", "nesterov"};
    static const char *linear[] = {"n_in", "n_out", "x_dtype", "y_dtype", "relu"};
    for (int i = 0; i < kMatrixNames; ++i) g_matrix_names[i] = PyUnicode_InternFromString(matrix[i]);
    for (int i = 0; i < kMuonNames; ++i) g_muon_names[i] = PyUnicode_InternFromString(muon[i]);
    for (int i = 0; i < kLinearNames; ++i) g_linear_names[i] = PyUnicode_InternFromString(linear[i]);
    static const char *norm[] = {"cols", "x_dtype", "y_dtype"};
    static const char *adapter[] = {"count", "rank", "n_in", "n_out", "dtype", "x_dtype", "y_dtype", "relu"};
    for (int i = 0; i < kNormNames; ++i) g_norm_names[i] = PyUnicode_InternFromString(norm[i]);
    for (int i = 0; i < kAdapterNames; ++i) g_adapter_names[i] = PyUnicode_InternFromString(adapter[i]);
    g_eps_name = PyUnicode_InternFromString("eps");
    return PyModule_Create(&g_module);
}

// Native marshalling of the few-bit serving calls (include/mpq.h, "Serving in few bits"): torch tensors in,
// C-ABI calls out.  A decode step makes these calls one after another with a few microseconds of work
// in each, and checking the tensors and allocating outputs through Python costs more than that; here it
// costs about a microsecond.  No arithmetic, no kernels: the functions of libmpq.so are given by address
// (init), so that whichever build the program loaded is the one that runs.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <exception>

#include "mpq.h"

namespace {

decltype(&mpq_mx_quantize) f_mx_quantize;
decltype(&mpq_mx_dequantize) f_mx_dequantize;
decltype(&mpq_mx_linear) f_mx_linear;
decltype(&mpq_cache_write) f_cache_write;
decltype(&mpq_cache_read) f_cache_read;
decltype(&mpq_cache_attention) f_cache_attention;
decltype(&mpq_g4_quantize) f_g4_quantize;
decltype(&mpq_g4_dequantize) f_g4_dequantize;
decltype(&mpq_g4_linear) f_g4_linear, f_g4_linear_exact;
decltype(&mpq_rotate) f_rotate;
decltype(&mpq_pages_extend) f_pages_extend;
decltype(&mpq_pages_trim) f_pages_trim;
PyObject *raise_status;      // raise_status(status, name): the exception of a refused call

// An argument was refused: the Python error is set.
struct Refused {};

[[noreturn]] void refuse(PyObject *type, const char *fmt, const char *a, const char *b = "")
{
    PyErr_Format(type, fmt, a, b);
    throw Refused();
}

const char *dtype_name(at::ScalarType t)
{
    switch (t) {
    case at::kFloat: return "torch.float32";
    case at::kHalf: return "torch.float16";
    case at::kBFloat16: return "torch.bfloat16";
    case at::kByte: return "torch.uint8";
    case at::kInt: return "torch.int32";
    case at::kLong: return "torch.int64";
    default: return c10::toString(t);
    }
}

// What the tensors of one call have in common: they lie on one device, which is the current one when the
// call is made (stream), and those that it makes belong to the stream it runs on.
class Call {
public:
    const at::Tensor &tensor(PyObject *o, const char *name)
    {
        if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a torch tensor", name);
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda()) refuse(PyExc_ValueError, "%s must be a CUDA tensor", name);
        const int device = t.device().index();
        if (device_ < 0) device_ = device;
        if (device != device_)
            refuse(PyExc_ValueError, "%s must lie on the other tensors' device, %s", name,
                   ("cuda:" + std::to_string(device_) + ", is on cuda:" + std::to_string(device)).c_str());
        return t;
    }
    // The stream argument's handle (None: the current stream's).
    void *stream(PyObject *o)
    {
        const int current = c10::cuda::current_device();
        if (device_ != current)
            refuse(PyExc_ValueError, "the tensors lie on %s, the current device is %s",
                   ("cuda:" + std::to_string(device_)).c_str(), ("cuda:" + std::to_string(current)).c_str());
        cudaStream_t const here = c10::cuda::getCurrentCUDAStream().stream();
        if (o == Py_None) return here;
        PyObject *h = PyObject_GetAttrString(o, "cuda_stream");
        if (!h) throw Refused();
        void *s = PyLong_AsVoidPtr(h);
        Py_DECREF(h);
        if (PyErr_Occurred()) throw Refused();
        stream_ = static_cast<cudaStream_t>(s);
        elsewhere_ = stream_ != here;
        return s;
    }
    // An output, after stream: in memory of that stream (a block of the current stream's may still be in use
    // there), not given out again before what the current stream has been asked by then is done with it either.
    at::Tensor empty(at::IntArrayRef shape, at::ScalarType type) const
    {
        const c10::Device device(c10::kCUDA, (c10::DeviceIndex)device_);
        if (!elsewhere_) return at::Tensor(at::detail::empty_cuda(shape, type, device, std::nullopt));
        const c10::cuda::CUDAStream here = c10::cuda::getCurrentCUDAStream();
        const c10::cuda::CUDAStreamGuard guard(
            c10::cuda::getStreamFromExternal(stream_, (c10::DeviceIndex)device_));
        at::Tensor t(at::detail::empty_cuda(shape, type, device, std::nullopt));
        t.record_stream(here);
        return t;
    }

private:
    int device_ = -1;
    cudaStream_t stream_ = nullptr;      // where it is not the current one
    bool elsewhere_ = false;
};

std::string text(at::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + (s.size() == 1 ? ",)" : ")");
}

void need_shape(const at::Tensor &t, const char *name, at::IntArrayRef shape)
{
    if (t.sizes() != shape)
        refuse(PyExc_ValueError, "%s must have shape %s", name,
               (text(shape) + ", got " + text(t.sizes())).c_str());
}

// A contiguous CUDA tensor of a type (and, where there is one, a shape).
const at::Tensor &dense(Call &call, PyObject *o, const char *name, at::ScalarType type)
{
    const at::Tensor &t = call.tensor(o, name);
    if (t.scalar_type() != type)
        refuse(PyExc_TypeError, "%s must be %s", name,
               (std::string(dtype_name(type)) + ", got " + dtype_name(t.scalar_type())).c_str());
    if (!t.is_contiguous()) refuse(PyExc_ValueError, "%s must be contiguous", name);
    return t;
}
const at::Tensor &dense(Call &call, PyObject *o, const char *name, at::ScalarType type, at::IntArrayRef shape)
{
    const at::Tensor &t = dense(call, o, name, type);
    need_shape(t, name, shape);
    return t;
}

int type_of(at::ScalarType t, const char *name)
{
    if (t == at::kFloat) return MPQ_F32;
    if (t == at::kHalf) return MPQ_F16;
    if (t == at::kBFloat16) return MPQ_BF16;
    refuse(PyExc_TypeError, "%s must be torch.float32, torch.float16 or torch.bfloat16, got %s", name,
           dtype_name(t));
}

at::ScalarType dtype_arg(PyObject *o)
{
    if (!THPDtype_Check(o)) refuse(PyExc_TypeError, "%s must be a torch.dtype", "dtype");
    const at::ScalarType t = reinterpret_cast<THPDtype *>(o)->scalar_type;
    type_of(t, "dtype");
    return t;
}

// A layout's struct: a ctypes Structure's memory.
template <typename L>
const L &layout(PyObject *o, const char *name)
{
    Py_buffer v;
    if (PyObject_GetBuffer(o, &v, PyBUF_SIMPLE) != 0) throw Refused();
    const L *p = v.len == (Py_ssize_t)sizeof(L) ? static_cast<const L *>(v.buf) : nullptr;
    PyBuffer_Release(&v);            // (the memory is the object's, which the caller holds)
    if (!p) refuse(PyExc_TypeError, "%s is not a layout of this kind", name);
    return *p;
}

long long integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    return v;
}

int integer32(PyObject *o, const char *name)
{
    const long long v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) refuse(PyExc_ValueError, "%s does not fit 32 bits", name);
    return (int)v;
}

// Row stride of a matrix [rows][d] with contiguous rows that do not overlap.
long long rows_of(const at::Tensor &t, const char *name, long long rows, long long d)
{
    need_shape(t, name, {rows, d});
    const long long step = t.stride(0);
    if ((t.stride(1) != 1 && d > 1) || (step < d && rows > 1))
        refuse(PyExc_ValueError, "%s must have contiguous rows that do not overlap", name);
    return step > d ? step : d;
}

template <typename L_>
const at::Tensor &packed(Call &call, PyObject *o, const char *name, const L_ &L)
{
    const at::Tensor &t = dense(call, o, name, at::kByte);
    if ((size_t)t.numel() < L.bytes)
        refuse(PyExc_ValueError, "%s is smaller than layout.bytes = %s", name,
               std::to_string(L.bytes).c_str());
    return t;
}

// One call of the library, other Python threads running meanwhile (a launch waits while its stream's queue is
// full, and what is ahead in the queue may need Python).
template <typename F, typename... A>
void run(const char *name, F f, A... args)
{
    mpq_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f(args...);
    Py_END_ALLOW_THREADS
    if (st == MPQ_OK) return;
    PyObject *r = PyObject_CallFunction(raise_status, "is", (int)st, name);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, name);
    throw Refused();
}

PyObject *same(PyObject *o)
{
    Py_INCREF(o);
    return o;
}

// --- the calls (arguments by position, all of them) ----------------------------------------------

PyObject *mx_quantize(PyObject *const *v)     // X, layout, packed, stream
{
    Call call;
    const at::Tensor &X = call.tensor(v[0], "X");
    const mpq_mx_matrix &L = layout<mpq_mx_matrix>(v[1], "layout");
    const long long ld = rows_of(X, "X", L.rows, L.d);
    const int type = type_of(X.scalar_type(), "X");
    const bool own = v[2] == Py_None;
    if (!own) packed(call, v[2], "packed", L);
    void *const stream = call.stream(v[3]);
    const at::Tensor out = own ? call.empty({(long long)L.bytes}, at::kByte) : THPVariable_Unpack(v[2]);
    run("mpq_mx_quantize", f_mx_quantize, X.data_ptr(), type, ld, &L, out.data_ptr(), stream);
    return own ? THPVariable_Wrap(out) : same(v[2]);
}

PyObject *mx_dequantize(PyObject *const *v)   // packed, layout, dtype, Y, stream
{
    Call call;
    const mpq_mx_matrix &L = layout<mpq_mx_matrix>(v[1], "layout");
    const at::Tensor &p = packed(call, v[0], "packed", L);
    const bool own = v[3] == Py_None;
    if (!own) call.tensor(v[3], "Y");
    void *const stream = call.stream(v[4]);
    const at::Tensor Y = own ? call.empty({L.rows, L.d}, dtype_arg(v[2])) : THPVariable_Unpack(v[3]);
    const long long ld = rows_of(Y, "Y", L.rows, L.d);
    run("mpq_mx_dequantize", f_mx_dequantize, p.data_ptr(), &L, Y.data_ptr(), type_of(Y.scalar_type(), "Y"),
        ld, stream);
    return own ? THPVariable_Wrap(Y) : same(v[3]);
}

PyObject *mx_linear(PyObject *const *v)       // X, x_layout, W, w_layout, bias, dtype, Y, stream
{
    Call call;
    const mpq_mx_matrix &xl = layout<mpq_mx_matrix>(v[1], "x_layout");
    const mpq_mx_matrix &wl = layout<mpq_mx_matrix>(v[3], "w_layout");
    const at::Tensor &X = packed(call, v[0], "X", xl), &W = packed(call, v[2], "W", wl);
    const at::Tensor *const bias = v[4] == Py_None ? nullptr : &dense(call, v[4], "bias", at::kFloat, {wl.rows});
    const bool own = v[6] == Py_None;
    if (!own) call.tensor(v[6], "Y");
    void *const stream = call.stream(v[7]);
    const at::Tensor Y = own ? call.empty({xl.rows, wl.rows}, dtype_arg(v[5])) : THPVariable_Unpack(v[6]);
    const long long ld = rows_of(Y, "Y", xl.rows, wl.rows);
    run("mpq_mx_linear", f_mx_linear, &xl, X.data_ptr(), &wl, W.data_ptr(), bias ? bias->data_ptr<float>() :
        nullptr, Y.data_ptr(), type_of(Y.scalar_type(), "Y"), ld, stream);
    return own ? THPVariable_Wrap(Y) : same(v[6]);
}

// A cache's codes and scales.
struct Storage {
    const at::Tensor &codes, &scales;
    Storage(Call &call, const mpq_kv_cache &L, PyObject *c, PyObject *s)
        : codes(dense(call, c, "codes", at::kByte, {L.pages, 2, L.heads, L.page, L.row_bytes})),
          scales(dense(call, s, "scales", at::kFloat, {L.pages, 2, L.heads, L.page}))
    {
    }
};

const at::Tensor &slots_arg(Call &call, PyObject *o)
{
    const at::Tensor &t = dense(call, o, "slots", at::kLong);
    if (t.dim() != 1) refuse(PyExc_ValueError, "%s must be [T]", "slots");
    if (t.numel() > INT32_MAX) refuse(PyExc_ValueError, "%s has too many entries", "slots");
    return t;
}

PyObject *cache_write(PyObject *const *v)     // K, V, slots, layout, codes, scales, stream
{
    Call call;
    const at::Tensor &K = call.tensor(v[0], "K"), &V = call.tensor(v[1], "V"), &slots = slots_arg(call, v[2]);
    const mpq_kv_cache &L = layout<mpq_kv_cache>(v[3], "layout");
    const long long T = slots.numel();
    need_shape(K, "K", {T, L.heads, L.dim});
    need_shape(V, "V", {T, L.heads, L.dim});
    // (a dimension of one entry has no stride to speak of)
    long long ld[2];
    bool same_rows = K.scalar_type() == V.scalar_type();
    for (int i = 0; i < 2; ++i) {
        ld[i] = K.size(i) > 1 ? K.stride(i) : 0;
        same_rows = same_rows && ld[i] == (V.size(i) > 1 ? V.stride(i) : 0);
    }
    if (!same_rows) refuse(PyExc_ValueError, "K and V must have one type and the same strides%s", "");
    if (K.stride(2) != 1 || V.stride(2) != 1) refuse(PyExc_ValueError, "%s must have contiguous rows", "K and V");
    const Storage s(call, L, v[4], v[5]);
    void *const stream = call.stream(v[6]);
    run("mpq_cache_write", f_cache_write, K.data_ptr(), V.data_ptr(), type_of(K.scalar_type(), "K"), ld[0],
        ld[1], (int)T, slots.data_ptr<int64_t>(), &L, s.codes.data_ptr(), s.scales.data_ptr<float>(), stream);
    Py_RETURN_NONE;
}

PyObject *cache_read(PyObject *const *v)      // slots, layout, codes, scales, dtype, K, V, stream
{
    Call call;
    const at::Tensor &slots = slots_arg(call, v[0]);
    const mpq_kv_cache &L = layout<mpq_kv_cache>(v[1], "layout");
    const int64_t shape[3] = {slots.numel(), L.heads, L.dim};
    const Storage s(call, L, v[2], v[3]);
    const at::ScalarType type = v[5] == Py_None ? dtype_arg(v[4]) : call.tensor(v[5], "K").scalar_type();
    const int number = type_of(type, "K");
    for (int i = 0; i < 2; ++i)
        if (v[5 + i] != Py_None) dense(call, v[5 + i], i ? "V" : "K", type, shape);
    void *const stream = call.stream(v[7]);
    at::Tensor out[2];
    for (int i = 0; i < 2; ++i)
        out[i] = v[5 + i] == Py_None ? call.empty(shape, type) : THPVariable_Unpack(v[5 + i]);
    run("mpq_cache_read", f_cache_read, slots.data_ptr<int64_t>(), (int)shape[0], &L, s.codes.data_ptr(),
        s.scales.data_ptr<float>(), out[0].data_ptr(), out[1].data_ptr(), number, stream);
    PyObject *k = v[5] == Py_None ? THPVariable_Wrap(out[0]) : same(v[5]);
    PyObject *w = k ? (v[6] == Py_None ? THPVariable_Wrap(out[1]) : same(v[6])) : nullptr;
    PyObject *both = w ? PyTuple_Pack(2, k, w) : nullptr;
    Py_XDECREF(k);
    Py_XDECREF(w);
    return both;
}

// Q, table, lens, layout, codes, scales, scale, window, O, lse, workspace, stream
PyObject *cache_attention(PyObject *const *v)
{
    Call call;
    const at::Tensor &Q = call.tensor(v[0], "Q"), &table = dense(call, v[1], "table", at::kInt);
    const mpq_kv_cache &L = layout<mpq_kv_cache>(v[3], "layout");
    if (table.dim() != 2) refuse(PyExc_ValueError, "%s must be [B][columns]", "table");
    const long long B = table.size(0), cols = table.size(1);
    if (Q.dim() != 3 || Q.size(0) != B || Q.size(2) != L.dim)
        refuse(PyExc_ValueError, "Q must have shape (%s, got %s",
               (std::to_string(B) + ", q_heads, " + std::to_string(L.dim) + ")").c_str(),
               text(Q.sizes()).c_str());
    const long long q_heads = Q.size(1);
    if (Q.stride(2) != 1 || (q_heads > 1 && Q.stride(1) != L.dim))
        refuse(PyExc_ValueError, "%s must have consecutive heads", "Q");
    if (B > INT32_MAX || cols > INT32_MAX || q_heads > INT32_MAX)
        refuse(PyExc_ValueError, "%s is too large", "table or Q");
    const at::Tensor &lens = dense(call, v[2], "lens", at::kInt, {B});
    const Storage s(call, L, v[4], v[5]);
    const int type = type_of(Q.scalar_type(), "Q");
    const bool own = v[8] == Py_None;
    if (!own) dense(call, v[8], "O", Q.scalar_type(), Q.sizes());
    const at::Tensor *const lse = v[9] == Py_None ? nullptr : &dense(call, v[9], "lse", at::kFloat, {B, q_heads});
    const at::Tensor *const ws = v[10] == Py_None ? nullptr : &dense(call, v[10], "workspace", at::kByte);
    double scale = 1.0 / std::sqrt((double)L.dim);
    if (v[6] != Py_None) {
        scale = PyFloat_AsDouble(v[6]);
        if (scale == -1.0 && PyErr_Occurred()) throw Refused();
    }
    const int window = integer32(v[7], "window");
    void *const stream = call.stream(v[11]);
    const at::Tensor O = own ? call.empty(Q.sizes(), Q.scalar_type()) : THPVariable_Unpack(v[8]);
    run("mpq_cache_attention", f_cache_attention, Q.data_ptr(), type, Q.stride(0), (int)B, (int)q_heads, &L,
        s.codes.data_ptr(), s.scales.data_ptr<float>(), table.data_ptr<int>(), (int)cols, lens.data_ptr<int>(),
        (float)scale, window, O.data_ptr(), lse ? lse->data_ptr<float>() : nullptr, ws ? ws->data_ptr() :
        nullptr, ws ? (size_t)ws->numel() : 0, stream);
    return own ? THPVariable_Wrap(O) : same(v[8]);
}

PyObject *g4_quantize(PyObject *const *v)     // X, layout, packed, stream
{
    Call call;
    const at::Tensor &X = call.tensor(v[0], "X");
    const mpq_g4_matrix &L = layout<mpq_g4_matrix>(v[1], "layout");
    const long long ld = rows_of(X, "X", L.rows, L.d);
    const int type = type_of(X.scalar_type(), "X");
    const bool own = v[2] == Py_None;
    if (!own) packed(call, v[2], "packed", L);
    void *const stream = call.stream(v[3]);
    const at::Tensor out = own ? call.empty({(long long)L.bytes}, at::kByte) : THPVariable_Unpack(v[2]);
    run("mpq_g4_quantize", f_g4_quantize, X.data_ptr(), type, ld, &L, out.data_ptr(), stream);
    return own ? THPVariable_Wrap(out) : same(v[2]);
}

PyObject *g4_dequantize(PyObject *const *v)   // packed, layout, dtype, Y, stream
{
    Call call;
    const mpq_g4_matrix &L = layout<mpq_g4_matrix>(v[1], "layout");
    const at::Tensor &p = packed(call, v[0], "packed", L);
    const bool own = v[3] == Py_None;
    if (!own) call.tensor(v[3], "Y");
    void *const stream = call.stream(v[4]);
    const at::Tensor Y = own ? call.empty({L.rows, L.d}, dtype_arg(v[2])) : THPVariable_Unpack(v[3]);
    const long long ld = rows_of(Y, "Y", L.rows, L.d);
    run("mpq_g4_dequantize", f_g4_dequantize, p.data_ptr(), &L, Y.data_ptr(), type_of(Y.scalar_type(), "Y"), ld,
        stream);
    return own ? THPVariable_Wrap(Y) : same(v[3]);
}

bool flag(PyObject *o)
{
    const int r = PyObject_IsTrue(o);
    if (r < 0) throw Refused();
    return r != 0;
}

PyObject *g4_linear(PyObject *const *v)       // X, W, w_layout, bias, dtype, Y, stream, exact
{
    Call call;
    const bool exact = flag(v[7]);
    const at::Tensor &X = call.tensor(v[0], "X");
    const mpq_g4_matrix &L = layout<mpq_g4_matrix>(v[2], "w_layout");
    if (X.dim() != 2) refuse(PyExc_ValueError, "%s must be [T][d]", "X");
    const long long T = X.size(0), ldx = rows_of(X, "X", T, L.d);
    if (T > INT32_MAX) refuse(PyExc_ValueError, "%s has too many rows", "X");
    const int type = type_of(X.scalar_type(), "X");
    const at::Tensor &W = packed(call, v[1], "W", L);
    const at::Tensor *const bias = v[3] == Py_None ? nullptr : &dense(call, v[3], "bias", at::kFloat, {L.rows});
    const bool own = v[5] == Py_None;
    if (!own) call.tensor(v[5], "Y");
    void *const stream = call.stream(v[6]);
    const at::Tensor Y = own ? call.empty({T, L.rows}, v[4] == Py_None ? X.scalar_type() : dtype_arg(v[4]))
                             : THPVariable_Unpack(v[5]);
    const long long ldy = rows_of(Y, "Y", T, L.rows);
    run(exact ? "mpq_g4_linear_exact" : "mpq_g4_linear", exact ? f_g4_linear_exact : f_g4_linear, X.data_ptr(), type, ldx, (int)T, &L, W.data_ptr(),
        bias ? bias->data_ptr<float>() : nullptr, Y.data_ptr(), type_of(Y.scalar_type(), "Y"), ldy, stream);
    return own ? THPVariable_Wrap(Y) : same(v[5]);
}

// Q or K [T][heads][dim] of a rotation, and where its output goes (None: allocated later).
struct Turned {
    const at::Tensor *x = nullptr;
    at::Tensor y;
    bool own = false;
    mpq_rotate_rows rows = {};

    Turned(Call &call, PyObject *in, PyObject *out, PyObject *weight, const char *name, const char *out_name,
           const char *weight_name)
    {
        if (in == Py_None) {
            if (out != Py_None || weight != Py_None)
                refuse(PyExc_ValueError, "%s or %s without what they are for", out_name, weight_name);
            return;
        }
        x = &call.tensor(in, name);
        if (x->dim() != 3) refuse(PyExc_ValueError, "%s must be [T][heads][dim]", name);
        if (x->size(2) > 1 && x->stride(2) != 1) refuse(PyExc_ValueError, "%s must have contiguous rows", name);
        if (x->size(1) > INT32_MAX) refuse(PyExc_ValueError, "%s has too many heads", name);
        if (weight != Py_None)
            rows.weight = dense(call, weight, weight_name, at::kFloat, {x->size(2)}).data_ptr<float>();
        own = out == Py_None;
        if (own) return;
        y = call.tensor(out, out_name);
        need_shape(y, out_name, x->sizes());
        if (y.scalar_type() != x->scalar_type())
            refuse(PyExc_TypeError, "%s must have the type of its input, %s", out_name, dtype_name(x->scalar_type()));
        if (y.size(2) > 1 && y.stride(2) != 1) refuse(PyExc_ValueError, "%s must have contiguous rows", out_name);
    }
    void finish(Call &call)
    {
        if (!x) return;
        if (own) y = call.empty(x->sizes(), x->scalar_type());
        rows.x = x->data_ptr();
        rows.y = y.data_ptr();
        rows.heads = (int)x->size(1);
        rows.ld_token = x->size(0) > 1 ? x->stride(0) : 0;
        rows.ld_head = x->size(1) > 1 ? x->stride(1) : 0;
        rows.ldy_token = y.size(0) > 1 ? y.stride(0) : 0;
        rows.ldy_head = y.size(1) > 1 ? y.stride(1) : 0;
    }
    PyObject *result(PyObject *out) const { return x && own ? THPVariable_Wrap(y) : same(out); }
};

// Q, K, positions, turns, norm, q_weight, k_weight, eps, neighbours, shift, Yq, Yk, stream
PyObject *rotate(PyObject *const *v)
{
    Call call;
    Turned q(call, v[0], v[10], v[5], "Q", "Yq", "q_weight"), k(call, v[1], v[11], v[6], "K", "Yk", "k_weight");
    if (!q.x) refuse(PyExc_TypeError, "%s must be a torch tensor", "Q");
    const long long T = q.x->size(0), dim = q.x->size(2);
    if (T > INT32_MAX || dim > INT32_MAX) refuse(PyExc_ValueError, "%s is too large", "Q");
    if (k.x && (k.x->size(0) != T || k.x->size(2) != dim || k.x->scalar_type() != q.x->scalar_type()))
        refuse(PyExc_ValueError, "K must have Q's tokens, dim and type%s", "");
    const at::Tensor &positions = dense(call, v[2], "positions", at::kInt, {T});
    const at::Tensor &turns = dense(call, v[3], "turns", at::kLong);
    if (turns.dim() != 1 || turns.numel() > INT32_MAX / 2) refuse(PyExc_ValueError, "%s must be [rot / 2]", "turns");
    const int type = type_of(q.x->scalar_type(), "Q");
    const double eps = PyFloat_AsDouble(v[7]);
    if (eps == -1.0 && PyErr_Occurred()) throw Refused();
    const int norm = flag(v[4]), neighbours = flag(v[8]), shift = integer32(v[9], "shift");
    void *const stream = call.stream(v[12]);
    q.finish(call);
    k.finish(call);
    run("mpq_rotate", f_rotate, &q.rows, k.x ? &k.rows : nullptr, type, (int)T, (int)dim, positions.data_ptr<int>(),
        shift, reinterpret_cast<const uint64_t *>(turns.data_ptr<int64_t>()), 2 * (int)turns.numel(), neighbours,
        norm, (float)eps, stream);
    PyObject *a = q.result(v[10]), *b = a ? k.result(v[11]) : nullptr, *both = b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return both;
}

// The state of a cache's requests: want (add or keep), lens, table, pool, count, and where new lengths and the new
// count go (None: in place).
struct Requests {
    const at::Tensor &want, &lens, &table, &pool, &count;
    const at::Tensor &new_lens, &new_count;

    Requests(Call &call, const char *name, PyObject *w, PyObject *l, PyObject *t, PyObject *p, PyObject *c,
             PyObject *nl, PyObject *nc)
        : want(dense(call, w, name, at::kInt)), lens(dense(call, l, "lens", at::kInt, want.sizes())),
          table(dense(call, t, "table", at::kInt)), pool(dense(call, p, "pool", at::kInt)),
          count(dense(call, c, "count", at::kInt, {2})),
          new_lens(nl == Py_None ? lens : dense(call, nl, "new_lens", at::kInt, want.sizes())),
          new_count(nc == Py_None ? count : dense(call, nc, "new_count", at::kInt, {2}))
    {
        if (want.dim() != 1) refuse(PyExc_ValueError, "%s must be [B]", name);
        if (table.dim() != 2 || table.size(0) != want.size(0))
            refuse(PyExc_ValueError, "table must have shape (%s, columns), got %s",
                   std::to_string(want.size(0)).c_str(), text(table.sizes()).c_str());
        if (pool.dim() != 1) refuse(PyExc_ValueError, "%s must be [pages]", "pool");
        if (want.size(0) > INT32_MAX || table.size(1) > INT32_MAX || pool.size(0) > INT32_MAX)
            refuse(PyExc_ValueError, "%s is too large", "table or pool");
    }
};

// add, lens, table, pool, count, page, N, new_lens, new_count, slots, positions, taken, stream
PyObject *pages_extend(PyObject *const *v)
{
    Call call;
    const Requests r(call, "add", v[0], v[1], v[2], v[3], v[4], v[7], v[8]);
    const int page = integer32(v[5], "page");
    const long long N = integer(v[6]), B = r.want.size(0);
    if (N < 0) refuse(PyExc_ValueError, "%s must not be negative", "N");
    const char *const names[3] = {"slots", "positions", "taken"};
    const at::ScalarType types[3] = {at::kLong, at::kInt, at::kInt};
    const long long sizes[3] = {N, N, B};
    for (int i = 0; i < 3; ++i)
        if (v[9 + i] != Py_None) dense(call, v[9 + i], names[i], types[i], {sizes[i]});
    void *const stream = call.stream(v[12]);
    at::Tensor out[3];
    for (int i = 0; i < 3; ++i)
        out[i] = v[9 + i] == Py_None ? call.empty({sizes[i]}, types[i]) : THPVariable_Unpack(v[9 + i]);
    run("mpq_pages_extend", f_pages_extend, r.want.data_ptr<int>(), (int)B, page, (int)r.table.size(1),
        r.lens.data_ptr<int>(), r.new_lens.data_ptr<int>(), r.table.data_ptr<int>(), r.pool.data_ptr<int>(),
        (int)r.pool.size(0), r.count.data_ptr<int>(), r.new_count.data_ptr<int>(), out[0].data_ptr<int64_t>(),
        out[1].data_ptr<int>(), N, out[2].data_ptr<int>(), stream);
    PyObject *all = PyTuple_New(3);
    for (int i = 0; all && i < 3; ++i) {
        PyObject *o = v[9 + i] == Py_None ? THPVariable_Wrap(out[i]) : same(v[9 + i]);
        if (!o) {
            Py_DECREF(all);
            return nullptr;
        }
        PyTuple_SET_ITEM(all, i, o);
    }
    return all;
}

// keep, lens, table, pool, count, page, new_lens, new_count, stream
PyObject *pages_trim(PyObject *const *v)
{
    Call call;
    const Requests r(call, "keep", v[0], v[1], v[2], v[3], v[4], v[6], v[7]);
    const int page = integer32(v[5], "page");
    void *const stream = call.stream(v[8]);
    run("mpq_pages_trim", f_pages_trim, r.want.data_ptr<int>(), (int)r.want.size(0), page, (int)r.table.size(1),
        r.lens.data_ptr<int>(), r.new_lens.data_ptr<int>(), r.table.data_ptr<int>(), r.pool.data_ptr<int>(),
        (int)r.pool.size(0), r.count.data_ptr<int>(), r.new_count.data_ptr<int>(), stream);
    Py_RETURN_NONE;
}

// No C++ exception leaves a call: refusals have their Python error set, others become RuntimeError.
template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyObject *guarded(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    if (n != N) return PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", N, n);
    try {
        return F(v);
    } catch (const Refused &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// init(raise_status, {name: address}): the library's functions.
PyObject *init(PyObject *, PyObject *args)
{
    PyObject *raise, *table;
    if (!PyArg_ParseTuple(args, "OO!", &raise, &PyDict_Type, &table)) return nullptr;
    bool ok = true;
    auto take = [&](auto &f, const char *name) {
        PyObject *a = PyDict_GetItemString(table, name);
        void *p = a ? PyLong_AsVoidPtr(a) : nullptr;
        if (!p) ok = false;
        f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(p);
    };
    take(f_mx_quantize, "mpq_mx_quantize");
    take(f_mx_dequantize, "mpq_mx_dequantize");
    take(f_mx_linear, "mpq_mx_linear");
    take(f_cache_write, "mpq_cache_write");
    take(f_cache_read, "mpq_cache_read");
    take(f_cache_attention, "mpq_cache_attention");
    take(f_g4_quantize, "mpq_g4_quantize");
    take(f_g4_dequantize, "mpq_g4_dequantize");
    take(f_g4_linear, "mpq_g4_linear");
    take(f_g4_linear_exact, "mpq_g4_linear_exact");
    take(f_rotate, "mpq_rotate");
    take(f_pages_extend, "mpq_pages_extend");
    take(f_pages_trim, "mpq_pages_trim");
    if (!ok) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, "an entry point is missing");
        return nullptr;
    }
    Py_INCREF(raise);
    Py_XDECREF(raise_status);
    raise_status = raise;
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *const *), Py_ssize_t N>
PyMethodDef method(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<F, N>)),
            METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {{"init", init, METH_VARARGS, nullptr},
                         method<mx_quantize, 4>("mx_quantize"),
                         method<mx_dequantize, 5>("mx_dequantize"),
                         method<mx_linear, 8>("mx_linear"),
                         method<cache_write, 7>("cache_write"),
                         method<cache_read, 8>("cache_read"),
                         method<cache_attention, 12>("cache_attention"),
                         method<g4_quantize, 4>("g4_quantize"),
                         method<g4_dequantize, 5>("g4_dequantize"),
                         method<g4_linear, 8>("g4_linear"),
                         method<rotate, 13>("rotate"),
                         method<pages_extend, 13>("pages_extend"),
                         method<pages_trim, 9>("pages_trim"),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_serve_binding", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" PyMODINIT_FUNC PyInit__serve_binding(void) { return PyModule_Create(&module); }

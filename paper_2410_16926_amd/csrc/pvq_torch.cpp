// Native half of binding.py: takes torch tensors apart, allocates results and calls libpvq on the current
// stream.  What a call of a small matrix costs is host time (a kernel of 4 us behind 10 us of attribute
// lookups, ctypes conversions and 3 us for the stream object in Python; about 4 us from here, most of it the
// launch itself), so the whole way from the Python call to the C ABI is native.  Argument marshalling only.
//
// Every function returns its result, or the library's negative status as an int (binding.py raises PvqError
// from it).  The interpreter lock is released around the library call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "pvq.h"

namespace {

// raised as the named Python exception
struct bad_argument {
    PyObject *type;
    const char *text;
};

void *context(PyObject *o)
{
    if (o == Py_None) return nullptr;
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw bad_argument{nullptr, nullptr};
    return p;
}

const at::Tensor &tensor(PyObject *o)
{
    if (!THPVariable_Check(o)) throw bad_argument{PyExc_TypeError, "a torch tensor is wanted"};
    return THPVariable_Unpack(o);
}

void *data(const at::Tensor &t) { return t.unsafeGetTensorImpl()->mutable_data(); }

// the address of a tensor's data; None gives a null pointer
void *data_or_null(PyObject *o) { return o == Py_None ? nullptr : data(tensor(o)); }

int64_t number(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw bad_argument{nullptr, nullptr};
    return v;
}

int dtype_code(at::ScalarType t)
{
    switch (t) {
    case at::kFloat: return PVQ_F32;
    case at::kHalf: return PVQ_F16;
    case at::kBFloat16: return PVQ_BF16;
    default: throw bad_argument{PyExc_KeyError, "a dtype of float32, float16 or bfloat16 is wanted"};
    }
}

// a dtype argument, or `otherwise` for None
at::ScalarType scalar_type(PyObject *o, at::ScalarType otherwise)
{
    if (o == Py_None) return otherwise;
    if (!THPDtype_Check(o)) throw bad_argument{PyExc_TypeError, "a torch dtype is wanted"};
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

at::Tensor new_tensor(at::IntArrayRef shape, at::ScalarType type, const at::Tensor &like)
{
    return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
}

// rows, columns and row stride of a matrix with unit column stride; a single row is as long as it is wide
struct matrix_shape {
    int64_t rows, cols, ld;
};
matrix_shape matrix(const at::Tensor &t)
{
    if (t.dim() != 2) throw bad_argument{PyExc_ValueError, "a matrix is wanted"};
    return {t.size(0), t.size(1), t.size(0) > 1 ? t.stride(0) : std::max<int64_t>(t.size(1), 1)};
}

void *current_stream() { return (void *)c10::hip::getCurrentHIPStream().stream(); }

struct without_lock {
    PyThreadState *state = PyEval_SaveThread();
    ~without_lock() { PyEval_RestoreThread(state); }
};

PyObject *status_or(int status, const at::Tensor &result)
{
    return status ? PyLong_FromLong(status) : THPVariable_Wrap(result);
}

// ---- packed planes -----------------------------------------------------------------------------------

struct planes {
    at::Tensor index, scale, rownorm;
};

// the planes of rows x cols for a context, or a negative status
int new_planes(const pvq_ctx *c, int64_t rows, int64_t cols, const at::Tensor &like, planes &p)
{
    size_t index_bytes = 0, scale_bytes = 0;
    int D = 0, scale_bits = 0;
    int status = pvq_packed_sizes(c, rows, cols, &index_bytes, &scale_bytes, nullptr);
    if (!status) status = pvq_ctx_info(c, &D, nullptr, nullptr, &scale_bits);
    if (status) return status;
    const int64_t n = std::max<int64_t>(rows, 1);
    p.index = new_tensor({rows, (int64_t)index_bytes / 4 / n}, at::kInt, like);
    p.scale = scale_bits ? new_tensor({rows, (int64_t)scale_bytes / 4 / n}, at::kInt, like)
                         : new_tensor({rows, cols / D}, at::kFloat, like);
    p.rownorm = new_tensor({rows}, at::kFloat, like);
    return PVQ_OK;
}

PyObject *wrap(const planes &p)
{
    PyObject *index = THPVariable_Wrap(p.index), *scale = THPVariable_Wrap(p.scale), *rownorm = THPVariable_Wrap(p.rownorm);
    PyObject *r = index && scale && rownorm ? PyTuple_Pack(3, index, scale, rownorm) : nullptr;
    Py_XDECREF(index); Py_XDECREF(scale); Py_XDECREF(rownorm);
    return r;
}

// ---- the calls ---------------------------------------------------------------------------------------

// (ctx, W, index, scale, rownorm, pulses): planes given, or None for new ones.  Returns None where the planes were
// given, else the three new ones.
PyObject *encode(PyObject *const *a)
{
    const pvq_ctx *c = (const pvq_ctx *)context(a[0]);
    const at::Tensor &W = tensor(a[1]);
    const matrix_shape m = matrix(W);
    const int dtype = dtype_code(W.scalar_type());
    const bool given = a[2] != Py_None;
    planes p;
    if (!given)
        if (const int status = new_planes(c, m.rows, m.cols, W, p)) return PyLong_FromLong(status);
    void *index = given ? data(tensor(a[2])) : data(p.index), *scale = given ? data_or_null(a[3]) : data(p.scale);
    void *rownorm = given ? data_or_null(a[4]) : data(p.rownorm), *pulses = data_or_null(a[5]);
    void *w = data(W), *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_encode(c, w, dtype, m.rows, m.cols, m.ld, (uint32_t *)index, scale, (float *)rownorm, (int8_t *)pulses, stream);
    }
    if (status) return PyLong_FromLong(status);
    if (given) Py_RETURN_NONE;
    return wrap(p);
}

// (ctx, X, block, signs, index, scale, rownorm)
PyObject *rotate_encode(PyObject *const *a)
{
    const pvq_ctx *c = (const pvq_ctx *)context(a[0]);
    const at::Tensor &X = tensor(a[1]);
    const matrix_shape m = matrix(X);
    const int dtype = dtype_code(X.scalar_type()), block = (int)number(a[2]);
    const bool given = a[4] != Py_None;
    planes p;
    if (!given)
        if (const int status = new_planes(c, m.rows, m.cols, X, p)) return PyLong_FromLong(status);
    void *index = given ? data(tensor(a[4])) : data(p.index), *scale = given ? data_or_null(a[5]) : data(p.scale);
    void *rownorm = given ? data_or_null(a[6]) : data(p.rownorm);
    void *x = data(X), *signs = data_or_null(a[3]), *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_rotate_encode(c, x, dtype, m.rows, m.cols, m.ld, block, (const uint8_t *)signs, (uint32_t *)index, scale, (float *)rownorm, stream);
    }
    if (status) return PyLong_FromLong(status);
    if (given) Py_RETURN_NONE;
    return wrap(p);
}

// (ctx, index, scale, rownorm, rows, cols, out_dtype or None, out or None)
PyObject *decode(PyObject *const *a)
{
    const pvq_ctx *c = (const pvq_ctx *)context(a[0]);
    const at::Tensor &index = tensor(a[1]);
    const int64_t rows = number(a[4]), cols = number(a[5]);
    const at::Tensor out = a[7] != Py_None ? tensor(a[7]) : new_tensor({rows, cols}, scalar_type(a[6], at::kFloat), index);
    const int dtype = dtype_code(out.scalar_type());
    const int64_t ld = rows > 1 ? out.stride(0) : std::max<int64_t>(cols, 1);
    void *i = data(index), *scale = data_or_null(a[2]), *rownorm = data_or_null(a[3]), *o = data(out), *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_decode(c, (const uint32_t *)i, scale, (const float *)rownorm, rows, cols, o, dtype, ld, stream);
    }
    return status_or(status, out);
}

// (ctx, index, scale, rownorm, rows, cols, x, out or None)
PyObject *decode_gemv(PyObject *const *a)
{
    const pvq_ctx *c = (const pvq_ctx *)context(a[0]);
    const at::Tensor &index = tensor(a[1]), &x = tensor(a[6]);
    const int64_t rows = number(a[4]), cols = number(a[5]);
    if (x.dim() != 2 || x.scalar_type() != at::kBFloat16 || x.size(1) != cols)
        throw bad_argument{PyExc_AssertionError, "x is bfloat16 [batch][cols]"};
    const int64_t batch = x.size(0);
    const at::Tensor out = a[7] != Py_None ? tensor(a[7]) : new_tensor({batch, rows}, at::kFloat, x);
    const int64_t ldx = batch > 1 ? x.stride(0) : std::max<int64_t>(cols, 1), ldy = batch > 1 ? out.stride(0) : std::max<int64_t>(rows, 1);
    void *i = data(index), *scale = data_or_null(a[2]), *rownorm = data_or_null(a[3]), *xp = data(x), *o = data(out), *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_decode_gemv(c, (const uint32_t *)i, scale, (const float *)rownorm, rows, cols, xp, (int)batch, ldx, (float *)o, ldy, stream);
    }
    return status_or(status, out);
}

// (X, block, signs, inverse, out or None, out_dtype or None)
PyObject *hadamard(PyObject *const *a)
{
    const at::Tensor &X = tensor(a[0]);
    if (X.dim() != 2) throw bad_argument{PyExc_ValueError, "a matrix is wanted"};
    const int64_t rows = X.size(0), cols = X.size(1);
    const at::Tensor out = a[4] != Py_None ? tensor(a[4]) : new_tensor({rows, cols}, scalar_type(a[5], X.scalar_type()), X);
    const int in_dtype = dtype_code(X.scalar_type()), out_dtype = dtype_code(out.scalar_type()), block = (int)number(a[1]);
    const int inverse = PyObject_IsTrue(a[3]);
    if (inverse < 0) throw bad_argument{nullptr, nullptr};
    const int64_t ldx = rows > 1 ? X.stride(0) : cols, ldy = rows > 1 ? out.stride(0) : cols;
    void *x = data(X), *signs = data_or_null(a[2]), *o = data(out), *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_hadamard(x, in_dtype, rows, cols, ldx, block, (const uint8_t *)signs, inverse, o, out_dtype, ldy, stream);
    }
    return status_or(status, out);
}

// ---- 8-bit blocks ------------------------------------------------------------------------------------
// These calls check what they are given: all tensors on one GPU, which is made the current one for the call (its current
// stream is used), block planes of the shapes that their matrix has, matrices of floats with unit column stride.

struct blocks {
    at::Tensor codes, exps;
    const uint8_t *c() const { return (const uint8_t *)data(codes); }
    const uint8_t *e() const { return (const uint8_t *)data(exps); }
    uint8_t *c() { return (uint8_t *)data(codes); }
    uint8_t *e() { return (uint8_t *)data(exps); }
};

int64_t code_row(int64_t cols) { return (cols + 127) / 128 * 128; }
int64_t exp_row(int64_t cols) { return (code_row(cols) / 128 + 3) / 4 * 4; }

// the first tensor's device, or an error
at::Device gpu_of(const at::Tensor &t)
{
    if (!t.is_cuda()) throw bad_argument{PyExc_ValueError, "a tensor on the GPU is wanted"};
    return t.device();
}

void check_plane(const at::Tensor &t, int64_t rows, int64_t row, at::Device device)
{
    if (t.device() != device) throw bad_argument{PyExc_ValueError, "tensors on one GPU are wanted"};
    if (t.scalar_type() != at::kByte || t.dim() != 2 || t.size(0) != rows || t.size(1) != row || !t.is_contiguous())
        throw bad_argument{PyExc_ValueError, "contiguous uint8 planes [rows][128 ceil(cols/128)] and [rows][4 ceil(cols/512)] are wanted"};
}

blocks blocks_of(PyObject *codes, PyObject *exps, int64_t rows, int64_t cols, at::Device device)
{
    blocks b{tensor(codes), tensor(exps)};
    check_plane(b.codes, rows, code_row(cols), device);
    check_plane(b.exps, rows, exp_row(cols), device);
    return b;
}

blocks new_blocks(int64_t rows, int64_t cols, const at::Tensor &like)
{
    return {new_tensor({rows, code_row(cols)}, at::kByte, like), new_tensor({rows, exp_row(cols)}, at::kByte, like)};
}

PyObject *wrap(const blocks &b)
{
    PyObject *codes = THPVariable_Wrap(b.codes), *exps = THPVariable_Wrap(b.exps);
    PyObject *r = codes && exps ? PyTuple_Pack(2, codes, exps) : nullptr;
    Py_XDECREF(codes); Py_XDECREF(exps);
    return r;
}

struct floats {
    at::Tensor t;
    int dtype;
    int64_t ld;
    void *p() const { return data(t); }
};

floats floats_of(const at::Tensor &t, int64_t rows, int64_t cols, at::Device device)
{
    if (t.device() != device) throw bad_argument{PyExc_ValueError, "tensors on one GPU are wanted"};
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols) throw bad_argument{PyExc_ValueError, "a matrix of another shape is wanted"};
    if (cols > 1 && rows > 0 && t.stride(1) != 1) throw bad_argument{PyExc_ValueError, "a matrix with unit column stride is wanted"};
    if (rows > 1 && t.stride(0) < cols) throw bad_argument{PyExc_ValueError, "a matrix whose rows lie one behind the other is wanted"};
    return {t, dtype_code(t.scalar_type()), rows > 1 ? t.stride(0) : std::max<int64_t>(cols, 1)};
}

floats bf16_of(PyObject *o, int64_t rows, int64_t cols, at::Device device)
{
    const floats f = floats_of(tensor(o), rows, cols, device);
    if (f.dtype != PVQ_BF16) throw bad_argument{PyExc_ValueError, "a bfloat16 matrix is wanted"};
    return f;
}

// the given result, or a new one
floats result_of(PyObject *out, PyObject *out_dtype, int64_t rows, int64_t cols, const at::Tensor &like)
{
    return floats_of(out != Py_None ? tensor(out) : new_tensor({rows, cols}, scalar_type(out_dtype, at::kFloat), like), rows, cols, like.device());
}

// scratch memory of a call, from torch's allocator for the current stream
struct scratch {
    at::Tensor t;
    size_t bytes;
    scratch(size_t n, const at::Tensor &like) : bytes(n) { if (n) t = new_tensor({(int64_t)n}, at::kByte, like); }
    void *p() const { return bytes ? data(t) : nullptr; }
};

// (X, codes or None, exponents or None): the two planes
PyObject *fp8_encode(PyObject *const *a)
{
    const at::Tensor &X = tensor(a[0]);
    const at::Device device = gpu_of(X);
    if (X.dim() != 2) throw bad_argument{PyExc_ValueError, "a matrix is wanted"};
    const int64_t rows = X.size(0), cols = X.size(1);
    const floats x = floats_of(X, rows, cols, device);
    const c10::DeviceGuard guard(device);
    blocks b = a[1] != Py_None ? blocks_of(a[1], a[2], rows, cols, device) : new_blocks(rows, cols, X);
    void *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_fp8_encode(x.p(), x.dtype, rows, cols, x.ld, b.c(), b.e(), stream);
    }
    return status ? PyLong_FromLong(status) : wrap(b);
}

// (codes, exponents, rows, cols, out_dtype or None, out or None)
PyObject *fp8_decode(PyObject *const *a)
{
    const int64_t rows = number(a[2]), cols = number(a[3]);
    const at::Device device = gpu_of(tensor(a[0]));
    const blocks b = blocks_of(a[0], a[1], rows, cols, device);
    const c10::DeviceGuard guard(device);
    const floats y = result_of(a[5], a[4], rows, cols, b.codes);
    void *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_fp8_decode(b.c(), b.e(), rows, cols, y.p(), y.dtype, y.ld, stream);
    }
    return status_or(status, y.t);
}

// (codes and exponents of A, of B, m, n, k, out_dtype or None, out or None)
PyObject *fp8_product(PyObject *const *a)
{
    const int64_t m = number(a[4]), n = number(a[5]), k = number(a[6]);
    const at::Device device = gpu_of(tensor(a[0]));
    const blocks x = blocks_of(a[0], a[1], m, k, device), w = blocks_of(a[2], a[3], n, k, device);
    const c10::DeviceGuard guard(device);
    const floats y = result_of(a[8], a[7], m, n, x.codes);
    size_t bytes = 0;
    if (const int status = pvq_fp8_product_work_bytes(m, n, k, y.dtype, &bytes)) return PyLong_FromLong(status);
    const scratch work(bytes, x.codes);
    void *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_fp8_product(x.c(), x.e(), m, w.c(), w.e(), n, k, y.p(), y.dtype, y.ld, work.p(), bytes, stream);
    }
    return status_or(status, y.t);
}

// (dY, codes and exponents of W, m, n, k, out_dtype or None, out or None)
PyObject *fp8_input_grad(PyObject *const *a)
{
    const int64_t m = number(a[3]), n = number(a[4]), k = number(a[5]);
    const at::Device device = gpu_of(tensor(a[0]));
    const floats dy = bf16_of(a[0], m, n, device);
    const blocks w = blocks_of(a[1], a[2], n, k, device);
    const c10::DeviceGuard guard(device);
    const floats dx = result_of(a[7], a[6], m, k, w.codes);
    size_t bytes = 0;
    if (const int status = pvq_fp8_input_grad_work_bytes(dy.p(), dy.ld, m, n, k, &bytes)) return PyLong_FromLong(status);
    const scratch work(bytes, w.codes);
    void *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_fp8_input_grad(dy.p(), dy.ld, m, w.c(), w.e(), n, k, dx.p(), dx.dtype, dx.ld, work.p(), bytes, stream);
    }
    return status_or(status, dx.t);
}

// (dY, codes and exponents of X, m, n, k, out_dtype or None, out or None)
PyObject *fp8_weight_grad(PyObject *const *a)
{
    const int64_t m = number(a[3]), n = number(a[4]), k = number(a[5]);
    const at::Device device = gpu_of(tensor(a[0]));
    const floats dy = bf16_of(a[0], m, n, device);
    const blocks x = blocks_of(a[1], a[2], m, k, device);
    const c10::DeviceGuard guard(device);
    const floats dw = result_of(a[7], a[6], n, k, x.codes);
    size_t bytes = 0;
    if (const int status = pvq_fp8_weight_grad_work_bytes(dy.p(), dy.ld, m, n, k, &bytes)) return PyLong_FromLong(status);
    const scratch work(bytes, x.codes);
    void *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_fp8_weight_grad(dy.p(), dy.ld, m, n, x.c(), x.e(), k, dw.p(), dw.dtype, dw.ld, work.p(), bytes, stream);
    }
    return status_or(status, dw.t);
}

// (codes and exponents of X, gate, up, m, n, k, activation, out_dtype or None, out or None, whether H is wanted in blocks, whether
// G and U are kept): H (a tensor, or the two planes), or (H, G's planes, U's planes)
PyObject *fp8_gated(PyObject *const *a)
{
    const int64_t m = number(a[6]), n = number(a[7]), k = number(a[8]);
    const int act = (int)number(a[9]);
    const bool encoded = PyObject_IsTrue(a[12]) == 1, keep = PyObject_IsTrue(a[13]) == 1;
    const at::Device device = gpu_of(tensor(a[0]));
    const blocks x = blocks_of(a[0], a[1], m, k, device), gate = blocks_of(a[2], a[3], n, k, device), up = blocks_of(a[4], a[5], n, k, device);
    const c10::DeviceGuard guard(device);
    floats h{{}, PVQ_BF16, 0};
    blocks hb, g, u;
    if (encoded) hb = new_blocks(m, n, x.codes);
    else h = result_of(a[11], a[10], m, n, x.codes);
    if (keep) { g = new_blocks(m, n, x.codes); u = new_blocks(m, n, x.codes); }
    size_t bytes = 0;
    if (const int status = pvq_fp8_gated_work_bytes(m, n, k, h.dtype, encoded || keep, &bytes)) return PyLong_FromLong(status);
    const scratch work(bytes, x.codes);
    void *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_fp8_gated(x.c(), x.e(), m, gate.c(), gate.e(), up.c(), up.e(), n, k, act, encoded ? nullptr : h.p(), h.dtype, h.ld,
                               encoded ? hb.c() : nullptr, encoded ? hb.e() : nullptr, keep ? g.c() : nullptr, keep ? g.e() : nullptr,
                               keep ? u.c() : nullptr, keep ? u.e() : nullptr, work.p(), bytes, stream);
    }
    if (status) return PyLong_FromLong(status);
    PyObject *first = encoded ? wrap(hb) : THPVariable_Wrap(h.t);
    if (!keep || !first) return first;
    PyObject *second = wrap(g), *third = wrap(u);
    PyObject *r = second && third ? PyTuple_Pack(3, first, second, third) : nullptr;
    Py_DECREF(first); Py_XDECREF(second); Py_XDECREF(third);
    return r;
}

// (dH, codes and exponents of X, gate, up, G, U, m, n, k, activation, out_dtype or None, whether dX is wanted, whether dWg and dWu
// are): (dX or None, dWg or None, dWu or None)
PyObject *fp8_gated_backward(PyObject *const *a)
{
    const int64_t m = number(a[11]), n = number(a[12]), k = number(a[13]);
    const int act = (int)number(a[14]);
    const bool want_x = PyObject_IsTrue(a[16]) == 1, want_w = PyObject_IsTrue(a[17]) == 1;
    const at::Device device = gpu_of(tensor(a[0]));
    const floats dh = bf16_of(a[0], m, n, device);
    const blocks x = blocks_of(a[1], a[2], m, k, device), gate = blocks_of(a[3], a[4], n, k, device), up = blocks_of(a[5], a[6], n, k, device);
    const blocks g = blocks_of(a[7], a[8], m, n, device), u = blocks_of(a[9], a[10], m, n, device);
    const c10::DeviceGuard guard(device);
    const at::ScalarType type = scalar_type(a[15], at::kFloat);
    const int dtype = dtype_code(type);
    at::Tensor dx, dwg, dwu;
    if (want_x) dx = new_tensor({m, k}, type, x.codes);
    if (want_w) { dwg = new_tensor({n, k}, type, x.codes); dwu = new_tensor({n, k}, type, x.codes); }
    size_t bytes = 0;
    if (const int status = pvq_fp8_gated_backward_work_bytes(m, n, k, &bytes)) return PyLong_FromLong(status);
    const scratch work(bytes, x.codes);
    void *stream = current_stream();
    int status;
    {
        without_lock unlocked;
        status = pvq_fp8_gated_backward(dh.p(), dh.ld, x.c(), x.e(), m, gate.c(), gate.e(), up.c(), up.e(), n, k, g.c(), g.e(), u.c(), u.e(), act,
                                        want_x ? data(dx) : nullptr, k, want_w ? data(dwg) : nullptr, want_w ? data(dwu) : nullptr, k, dtype,
                                        work.p(), bytes, stream);
    }
    if (status) return PyLong_FromLong(status);
    PyObject *r = PyTuple_New(3);
    const at::Tensor *parts[3] = {want_x ? &dx : nullptr, want_w ? &dwg : nullptr, want_w ? &dwu : nullptr};
    for (int i = 0; r && i < 3; i++) {
        PyObject *o = parts[i] ? THPVariable_Wrap(*parts[i]) : Py_NewRef(Py_None);
        if (!o) { Py_CLEAR(r); break; }
        PyTuple_SET_ITEM(r, i, o);
    }
    return r;
}

// (): the current stream's handle
PyObject *stream(PyObject *const *) { return PyLong_FromVoidPtr(current_stream()); }

// ---- the module --------------------------------------------------------------------------------------

template <PyObject *(*F)(PyObject *const *), int N>
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    try {
        if (n != N) throw bad_argument{PyExc_TypeError, "wrong number of arguments"};
        return F(args);
    } catch (const bad_argument &e) {
        if (e.type) PyErr_SetString(e.type, e.text);        // (else the interpreter has its error already)
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

#define PVQ_METHOD(NAME, N) {#NAME, (PyCFunction)(void (*)(void))call<NAME, N>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {PVQ_METHOD(encode, 6), PVQ_METHOD(rotate_encode, 7), PVQ_METHOD(decode, 8), PVQ_METHOD(decode_gemv, 8),
                         PVQ_METHOD(hadamard, 6), PVQ_METHOD(stream, 0), PVQ_METHOD(fp8_encode, 3), PVQ_METHOD(fp8_decode, 6),
                         PVQ_METHOD(fp8_product, 9), PVQ_METHOD(fp8_input_grad, 8), PVQ_METHOD(fp8_weight_grad, 8),
                         PVQ_METHOD(fp8_gated, 14), PVQ_METHOD(fp8_gated_backward, 18), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pvq_torch", "libpvq's calls on torch tensors", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// What the module was built for, for build.py, which looks for this text in the file before the module is loaded.
extern "C" __attribute__((used, visibility("default"))) const char pvq_torch_built_for[] = PVQ_BUILT_FOR;

PyMODINIT_FUNC PyInit__pvq_torch(void) { return PyModule_Create(&module); }

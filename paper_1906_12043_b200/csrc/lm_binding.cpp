// Python binding of the language-model operators and of AdamW (include/cocod_lm.h, cocod_adamw.h): looks the tensors over, allocates results and scratch through
// torch and makes the C call on torch's current stream.  Marshalling only.  The same in Python and ctypes took 5 to 8 us a
// call, as long as the kernels of a small call themselves.
//
// Every function returns its result, or the library's error code as an int (the caller raises); a tensor that does not fit is a ValueError,
// and a result or scratch that torch has no room for its OutOfMemoryError.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/Context.h>
#include <ATen/MemoryOverlap.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <sstream>
#include <stdexcept>
#include <string>
#include <vector>

#include "cocod_adamw.h"
#include "cocod_lm.h"

namespace {

using at::Tensor;

struct Matrix {
    void *data;
    int64_t ld, stride;
};

[[noreturn]] void refuse(const char *name, const std::string &need, const Tensor &t)
{
    std::ostringstream s;
    s << name << ": need " << need << "; got " << t.sizes() << " " << t.scalar_type() << " on " << t.device() << ", strides " << t.strides();
    throw std::invalid_argument(s.str());
}
inline bool there(const Tensor &t, at::ScalarType type, int64_t device)
{
    return t.scalar_type() == type && t.is_cuda() && t.get_device() == device && t.layout() == at::kStrided;
}
std::string place(int64_t device) { return " on cuda:" + std::to_string(device) + " (the current device at creation)"; }

// An M x cols matrix: rows contiguous, not overlapping, starting at multiples of `align` bytes.
Matrix rows(const Tensor &t, const char *name, int64_t M, int64_t cols, at::ScalarType type, int64_t device, int64_t align)
{
    if (there(t, type, device) && t.dim() == 2 && t.size(0) == M && t.size(1) == cols) {
        const int64_t ld = M > 1 ? t.stride(0) : (cols + 15) / 16 * 16, size = t.element_size();
        const uint64_t at = reinterpret_cast<uint64_t>(t.data_ptr());
        if ((cols <= 1 || t.stride(1) == 1) && ld >= cols && at % align == 0 && (ld * size) % align == 0) return Matrix{t.data_ptr(), ld, 0};
    }
    refuse(name, std::to_string(M) + " x " + std::to_string(cols) + " " + c10::toString(type) + place(device) +
                     ", rows contiguous, not overlapping and starting at multiples of " + std::to_string(align) + " bytes", t);
}

// One n x k matrix per group.
Matrix groups(const Tensor &t, const char *name, int64_t G, int64_t n, int64_t k, at::ScalarType type, int64_t device)
{
    if (there(t, type, device) && t.dim() == 3 && t.size(0) == G && t.size(1) == n && t.size(2) == k) {
        const int64_t ld = n > 1 ? t.stride(1) : (k + 7) / 8 * 8, stride = G > 1 ? t.stride(0) : n * ld, size = t.element_size();
        const uint64_t at = reinterpret_cast<uint64_t>(t.data_ptr());
        if ((k <= 1 || t.stride(2) == 1) && ld >= k && stride >= (n - 1) * ld + k && at % 16 == 0 && (ld * size) % 16 == 0 && (stride * size) % 16 == 0)
            return Matrix{t.data_ptr(), ld, stride};
    }
    refuse(name, std::to_string(G) + " x " + std::to_string(n) + " x " + std::to_string(k) + " " + c10::toString(type) + place(device) +
                     ", rows contiguous, rows and groups not overlapping and starting at multiples of 16 bytes", t);
}

void *vector(const Tensor &t, const char *name, int64_t n, at::ScalarType type, int64_t device)
{
    if (there(t, type, device) && t.dim() == 1 && t.size(0) == n && (n <= 1 || t.stride(0) == 1)) return t.data_ptr();
    refuse(name, std::to_string(n) + " contiguous " + c10::toString(type) + place(device), t);
}

const Tensor &tensor(PyObject *o, const char *name, int64_t dims)
{
    if (!THPVariable_Check(o)) throw std::invalid_argument(std::string(name) + ": need a tensor");
    const Tensor &t = THPVariable_Unpack(o);
    if (dims >= 0 && t.dim() != dims) refuse(name, std::to_string(dims) + " dimensions", t);
    return t;
}

int64_t whole(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw std::runtime_error("");       // (Python's own error stands)
    return v;
}

// The operators' device; kernels are launched on the current one.
int64_t device(PyObject *o)
{
    const int64_t dev = whole(o), now = c10::cuda::current_device();
    if (dev != now)
        throw std::invalid_argument("the current device is cuda:" + std::to_string(now) + ", these operators were made on cuda:" + std::to_string(dev) +
                                    ": call them under torch.cuda.device(" + std::to_string(dev) + ")");
    return dev;
}

// A result that is given may not lie on an operand, which other thread blocks still read (seen where one begins at the other, or both are without
// gaps; rows of one buffer beside one another are fine).
void apart(const Tensor &out, const char *out_name, const Tensor &in, const char *name, bool same_is_fine = false)
{
    const bool begins = out.data_ptr() == in.data_ptr() && out.numel() > 0 && in.numel() > 0;
    const at::MemOverlapStatus s = at::get_overlap_status(out, in);
    const bool same = begins && out.sizes() == in.sizes() && out.strides() == in.strides();
    if (same && same_is_fine) return;
    if (begins || s == at::MemOverlapStatus::Full || s == at::MemOverlapStatus::Partial)
        throw std::invalid_argument(std::string(out_name) + ": lies on " + name);
}

// The same for an operand that may be None.
void apart(const Tensor &out, const char *out_name, PyObject *in, const char *name)
{
    if (in != Py_None) apart(out, out_name, tensor(in, name, -1), name);
}

// The result's type: the caller's choice (0 bf16, 1 fp32, -1 none), which has to be the type of a result that is given.
at::ScalarType result_type(PyObject *out, int64_t code, at::ScalarType usual)
{
    const at::ScalarType chosen = code == 0 ? at::kBFloat16 : code == 1 ? at::kFloat : usual;
    if (out == Py_None) return chosen;
    const at::ScalarType type = tensor(out, "out", -1).scalar_type();
    if ((type != at::kBFloat16 && type != at::kFloat) || (code >= 0 && type != chosen))
        throw std::invalid_argument("out: the result's type is bfloat16 or float32, and the one asked for");
    return type;
}
inline int type_code(at::ScalarType t) { return t == at::kFloat ? COCOD_F32 : COCOD_BF16; }
// (the allocation itself, without the dispatcher's way to it, 0.4 us, where nobody listens there: no mode of the dispatcher, and no filling of new memory)
inline Tensor fresh(const Tensor &like, at::IntArrayRef shape, at::ScalarType type)
{
    const at::Context &c = at::globalContext();
    if (c10::impl::TorchDispatchModeTLS::any_modes_set() || (c.deterministicAlgorithms() && c.deterministicFillUninitializedMemory()))
        return at::empty(shape, like.options().dtype(type));
    return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
}
// A contiguous part of a buffer, `at` bytes behind its start, as a tensor of its own.
inline Tensor part_of(const Tensor &buffer, int64_t at, at::IntArrayRef shape, at::ScalarType type)
{
    const caffe2::TypeMeta meta = c10::scalarTypeToTypeMeta(type);
    Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(buffer.storage()), buffer.key_set(), meta);
    t.unsafeGetTensorImpl()->set_storage_offset(at / (int64_t)meta.itemsize());
    t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
    return t;
}

inline cocod_stream_t current(int64_t device) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
inline PyObject *code_or(int rc, const Tensor &t) { return rc == COCOD_OK ? THPVariable_Wrap(t) : PyLong_FromLong(rc); }
// A tensor that was written: what autograd kept of it is not what is there now; it is told, as by an operation in place.
inline void written(PyObject *o)
{
    const Tensor &t = THPVariable_Unpack(o);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// A result that was given, which has been written.
inline PyObject *given(PyObject *o)
{
    written(o);
    Py_INCREF(o);
    return o;
}
inline PyObject *none()
{
    Py_INCREF(Py_None);
    return Py_None;
}

template <PyObject *(*F)(PyObject *const *), int N>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    try {
        if (n != N) throw std::invalid_argument("wrong number of arguments");
        return F(args);
    } catch (const std::invalid_argument &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const c10::OutOfMemoryError &e) {
        PyObject *torch = PyImport_ImportModule("torch"), *type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        if (type) PyErr_SetString(type, e.what_without_backtrace());
        Py_XDECREF(type);
        Py_XDECREF(torch);
    } catch (const std::exception &e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}
inline cocod_lm_handle *handle(PyObject *o)
{
    void *p = PyLong_AsVoidPtr(o);
    if (!p) {
        if (PyErr_Occurred()) throw std::runtime_error("");
        throw std::invalid_argument("the operators were destroyed");
    }
    return static_cast<cocod_lm_handle *>(p);
}

// (handle, device, a, w, offsets, out or None, type)
template <bool FORWARD> PyObject *rows_product(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]);
    const char *name = FORWARD ? "x" : "dy";
    const Tensor &x = tensor(a[2], name, 2), &w = tensor(a[3], "w", 3), &off = tensor(a[4], "offsets", 1);
    const int64_t G = w.size(0), n = w.size(1), k = w.size(2), M = x.size(0), cols = FORWARD ? n : k;
    const Matrix mx = rows(x, name, M, FORWARD ? k : n, at::kBFloat16, dev, 16), mw = groups(w, "w", G, n, k, at::kBFloat16, dev);
    const int32_t *offsets = static_cast<const int32_t *>(vector(off, "offsets", G + 1, at::kInt, dev));
    const at::ScalarType type = result_type(a[5], whole(a[6]), at::kBFloat16);
    const Tensor out = a[5] == Py_None ? fresh(x, {M, cols}, type) : tensor(a[5], "out", 2);
    const Matrix mo = a[5] == Py_None ? Matrix{out.data_ptr(), cols, 0} : rows(out, "out", M, cols, type, dev, 16);
    if (a[5] != Py_None) apart(out, "out", x, name), apart(out, "out", w, "w");
    const int rc = (FORWARD ? cocod_grouped_forward : cocod_grouped_input_grad)(h, (int)G, offsets, M, n, k, mx.data, mx.ld, mw.data, mw.ld, mw.stride,
                                                                               mo.data, mo.ld, type_code(type), current(dev));
    return rc == COCOD_OK && a[5] != Py_None ? given(a[5]) : code_or(rc, out);
}

// The result of a weight gradient: (tensor, its place, its type)
struct Weights {
    Tensor t;
    Matrix m;
    at::ScalarType type;
};
Weights weights(PyObject *out, PyObject *code, const Tensor &like, const char *name, int64_t G, int64_t n, int64_t k, at::ScalarType usual, int64_t dev)
{
    const at::ScalarType type = result_type(out, whole(code), usual);
    if (out != Py_None) {
        const Tensor &t = tensor(out, name, 3);
        return {t, groups(t, name, G, n, k, type, dev), type};
    }
    Tensor t = fresh(like, {G, n, k}, type);
    return {t, Matrix{t.data_ptr(), k, n * k}, type};
}

// (handle, device, dy, x, offsets, out or None, type)
PyObject *weight_grad(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]);
    const Tensor &dy = tensor(a[2], "dy", 2), &x = tensor(a[3], "x", 2), &off = tensor(a[4], "offsets", 1);
    const int64_t M = x.size(0), k = x.size(1), n = dy.size(1), G = off.size(0) - 1;
    const int32_t *offsets = static_cast<const int32_t *>(vector(off, "offsets", G + 1, at::kInt, dev));
    const Matrix md = rows(dy, "dy", M, n, at::kBFloat16, dev, 16), mx = rows(x, "x", M, k, at::kBFloat16, dev, 16);
    const Weights w = weights(a[5], a[6], dy, "out", G, n, k, at::kFloat, dev);
    if (a[5] != Py_None) apart(w.t, "out", dy, "dy"), apart(w.t, "out", x, "x");
    const int rc = cocod_grouped_weight_grad(h, (int)G, offsets, M, n, k, md.data, md.ld, mx.data, mx.ld, w.m.data, w.m.ld, w.m.stride, type_code(w.type),
                                             current(dev));
    return rc == COCOD_OK && a[5] != Py_None ? given(a[5]) : code_or(rc, w.t);
}

// (handle, device, dy, M, k, address, row stride, address of the scales, offsets, out or None, type, may take room)
PyObject *weight_grad_packed(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]), M = whole(a[3]), k = whole(a[4]);
    const Tensor &dy = tensor(a[2], "dy", 2), &off = tensor(a[8], "offsets", 1);
    const int64_t n = dy.size(1), G = off.size(0) - 1;
    const int32_t *offsets = static_cast<const int32_t *>(vector(off, "offsets", G + 1, at::kInt, dev));
    const Matrix md = rows(dy, "dy", M, n, at::kBFloat16, dev, 16);
    const Weights w = weights(a[9], a[10], dy, "out", G, n, k, at::kFloat, dev);
    if (a[9] != Py_None) apart(w.t, "out", dy, "dy");
    int64_t bytes = whole(a[11]) ? cocod_grouped_packed_workspace((int)G, M, n, k) : 0;
    Tensor scratch;
    if (bytes > 0) scratch = fresh(dy, {bytes}, at::kByte);
    else bytes = 0;
    const int rc = cocod_grouped_weight_grad_packed(h, (int)G, offsets, M, n, k, md.data, md.ld, static_cast<const int8_t *>(PyLong_AsVoidPtr(a[5])), whole(a[6]),
                                                    static_cast<const uint8_t *>(PyLong_AsVoidPtr(a[7])), w.m.data, w.m.ld, w.m.stride, type_code(w.type),
                                                    bytes ? scratch.data_ptr() : nullptr, bytes, current(dev));
    return rc == COCOD_OK && a[9] != Py_None ? given(a[9]) : code_or(rc, w.t);
}

// (handle, device, x): a new buffer with the whole numbers' rows and the scales;
// (handle, device, x, M, k, address, row stride, address of the scales): into a checkpoint that is there, whose shape has to be x's
PyObject *act_pack_new(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]);
    const Tensor &x = tensor(a[2], "x", 2);
    const int64_t M = x.size(0), k = x.size(1), ld = (k + 15) / 16 * 16;
    const Matrix mx = rows(x, "x", M, k, at::kBFloat16, dev, 1);
    const Tensor buffer = fresh(x, {M * ld + (k + 127) / 128 * M}, at::kByte);
    uint8_t *p = static_cast<uint8_t *>(buffer.data_ptr());
    return code_or(cocod_act_pack(h, M, k, mx.data, mx.ld, reinterpret_cast<int8_t *>(p), ld, p + M * ld, current(dev)), buffer);
}
PyObject *act_pack_into(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]), M = whole(a[3]), k = whole(a[4]);
    const Matrix mx = rows(tensor(a[2], "x", 2), "x", M, k, at::kBFloat16, dev, 1);
    return PyLong_FromLong(cocod_act_pack(h, M, k, mx.data, mx.ld, static_cast<int8_t *>(PyLong_AsVoidPtr(a[5])), whole(a[6]),
                                          static_cast<uint8_t *>(PyLong_AsVoidPtr(a[7])), current(dev)));
}

// (handle, device, a tensor of the checkpoint, M, k, address, row stride, address of the scales, out or None)
PyObject *act_unpack(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]), M = whole(a[3]), k = whole(a[4]);
    const Tensor out = a[8] == Py_None ? fresh(tensor(a[2], "checkpoint", -1), {M, k}, at::kBFloat16) : tensor(a[8], "out", 2);
    const Matrix mo = a[8] == Py_None ? Matrix{out.data_ptr(), k, 0} : rows(out, "out", M, k, at::kBFloat16, dev, 1);
    const int rc = cocod_act_unpack(h, M, k, static_cast<const int8_t *>(PyLong_AsVoidPtr(a[5])), whole(a[6]), static_cast<const uint8_t *>(PyLong_AsVoidPtr(a[7])),
                                    mo.data, mo.ld, current(dev));
    return rc == COCOD_OK && a[8] != Py_None ? given(a[8]) : code_or(rc, out);
}

// (handle, device, dh, M, k, address, row stride, out or None)
PyObject *act_relu_grad(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]), M = whole(a[3]), k = whole(a[4]);
    const Tensor &dh = tensor(a[2], "dh", 2);
    const Matrix md = rows(dh, "dh", M, k, at::kBFloat16, dev, 1);
    const Tensor out = a[7] == Py_None ? fresh(dh, {M, k}, at::kBFloat16) : tensor(a[7], "out", 2);
    const Matrix mo = a[7] == Py_None ? Matrix{out.data_ptr(), k, 0} : rows(out, "out", M, k, at::kBFloat16, dev, 1);
    if (a[7] != Py_None) apart(out, "out", dh, "dh", true);
    const int rc = cocod_act_relu_grad(h, M, k, md.data, md.ld, static_cast<const int8_t *>(PyLong_AsVoidPtr(a[5])), whole(a[6]), mo.data, mo.ld, current(dev));
    return rc == COCOD_OK && a[7] != Py_None ? given(a[7]) : code_or(rc, out);
}

// (handle, device, x, w, labels, offsets, row weights or None, limit [, dw or None, type])
template <bool GRAD> PyObject *vocab(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]), limit = whole(a[7]);
    const Tensor &x = tensor(a[2], "x", 2), &w = tensor(a[3], "w", 3);
    const int64_t G = w.size(0), V = w.size(1), D = w.size(2), M = x.size(0);
    const Matrix mx = rows(x, "x", M, D, at::kBFloat16, dev, 16), mw = groups(w, "w", G, V, D, at::kBFloat16, dev);
    const int32_t *labels = static_cast<const int32_t *>(vector(tensor(a[4], "labels", 1), "labels", M, at::kInt, dev));
    const int32_t *offsets = static_cast<const int32_t *>(vector(tensor(a[5], "offsets", 1), "offsets", G + 1, at::kInt, dev));
    const float *weight = a[6] == Py_None ? nullptr : static_cast<const float *>(vector(tensor(a[6], "row_weights", 1), "row_weights", M, at::kFloat, dev));
    Weights dw{};
    if (GRAD) dw = weights(a[8], a[9], x, "dw", G, V, D, at::kBFloat16, dev);
    if (GRAD && a[8] != Py_None) apart(dw.t, "dw", x, "x"), apart(dw.t, "dw", w, "w");
    const int64_t bytes = cocod_vocab_workspace((int)G, M, V, D, GRAD, GRAD ? type_code(dw.type) : COCOD_BF16, limit);
    if (bytes < 0) return PyLong_FromLong((long)bytes);
    const Tensor scratch = fresh(x, {bytes}, at::kByte), loss = fresh(x, {G}, at::kFloat), row_loss = fresh(x, {M}, at::kFloat);
    float *l = static_cast<float *>(loss.data_ptr()), *r = static_cast<float *>(row_loss.data_ptr());
    if (!GRAD) {
        const int rc = cocod_vocab_loss(h, (int)G, offsets, M, V, D, mx.data, mx.ld, mw.data, mw.ld, mw.stride, labels, weight, l, r, scratch.data_ptr(), bytes,
                                        current(dev));
        return rc == COCOD_OK ? Py_BuildValue("(NN)", THPVariable_Wrap(loss), THPVariable_Wrap(row_loss)) : PyLong_FromLong(rc);
    }
    const Tensor dx = fresh(x, {M, D}, at::kBFloat16);
    const int rc = cocod_vocab_loss_grad(h, (int)G, offsets, M, V, D, mx.data, mx.ld, mw.data, mw.ld, mw.stride, labels, weight, l, r, dx.data_ptr(), D,
                                         dw.m.data, dw.m.ld, dw.m.stride, type_code(dw.type), scratch.data_ptr(), bytes, current(dev));
    if (rc != COCOD_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NNNN)", THPVariable_Wrap(loss), THPVariable_Wrap(row_loss), THPVariable_Wrap(dx),
                         a[8] == Py_None ? THPVariable_Wrap(dw.t) : given(a[8]));
}

// ------------------------------------------------------------------------------------------ experts
// A tensor's type as the library names it: bf16 or fp32.
at::ScalarType value_type(const Tensor &t, const char *name)
{
    const at::ScalarType type = t.scalar_type();
    if (type != at::kBFloat16 && type != at::kFloat) refuse(name, "bfloat16 or float32", t);
    return type;
}
// T x k values side by side.
void *table(const Tensor &t, const char *name, int64_t T, int64_t k, at::ScalarType type, int64_t device)
{
    if (there(t, type, device) && t.dim() == 2 && t.size(0) == T && t.size(1) == k && t.is_contiguous()) return t.data_ptr();
    refuse(name, std::to_string(T) + " x " + std::to_string(k) + " contiguous " + c10::toString(type) + place(device), t);
}
// A matrix whose rows may start anywhere.  `given` (None: a new one like `like`) or a new one, which has to lie apart from the operands.
Matrix any_rows(const Tensor &t, const char *name, int64_t M, int64_t cols, at::ScalarType type, int64_t dev)
{
    if (there(t, type, dev) && t.dim() == 2 && t.size(0) == M && t.size(1) == cols && (cols <= 1 || t.stride(1) == 1)) {
        const int64_t ld = M > 1 ? t.stride(0) : cols;
        if (ld >= cols) return Matrix{t.data_ptr(), ld, 0};
    }
    refuse(name, std::to_string(M) + " x " + std::to_string(cols) + " " + c10::toString(type) + place(dev) + ", rows contiguous and not overlapping", t);
}

// (handle, device, experts, E): (offsets, counts, order, place, all four in one buffer)
PyObject *expert_sort(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]), E = whole(a[3]);
    const Tensor &e = tensor(a[2], "experts", 2);
    const int64_t T = e.size(0), k = e.size(1);
    const Matrix m = any_rows(e, "experts", T, k, at::kInt, dev);
    if (E < 1 || E > COCOD_LM_MAX_GROUPS || k < 1 || k > COCOD_LM_MAX_CHOICES)
        throw std::invalid_argument("experts: 1 to " + std::to_string(COCOD_LM_MAX_CHOICES) + " choices among 1 to " + std::to_string(COCOD_LM_MAX_GROUPS) + " experts");
    const int64_t bytes = cocod_expert_workspace(T, (int)k, (int)E);
    if (bytes < 0) return PyLong_FromLong((long)bytes);
    const int64_t N = T * k, at[5] = {0, E + 1, 2 * E + 1, 2 * E + 1 + N, 2 * E + 1 + 2 * N};      // offsets, counts, order, place, scratch
    const Tensor all = fresh(e, {at[4] + bytes / 4}, at::kInt);
    int32_t *p = static_cast<int32_t *>(all.data_ptr());
    const int rc = cocod_expert_sort(h, T, (int)k, (int)E, static_cast<const int32_t *>(m.data), m.ld, p, p + at[1], p + at[2], p + at[3], p + at[4], bytes, current(dev));
    if (rc != COCOD_OK) return PyLong_FromLong(rc);
    const auto part = [&](int i, at::IntArrayRef shape) { return THPVariable_Wrap(part_of(all, 4 * at[i], shape, at::kInt)); };
    return Py_BuildValue("(NNNN)", part(0, {E + 1}), part(1, {E}), part(2, {N}), part(3, {T, k}));
}

// (handle, device, x, place, out or None)
PyObject *expert_rows(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]);
    const Tensor &x = tensor(a[2], "x", 2), &at = tensor(a[3], "place", 2);
    const int64_t T = x.size(0), D = x.size(1), k = at.size(1);
    const at::ScalarType type = value_type(x, "x");
    const Matrix m = any_rows(x, "x", T, D, type, dev);
    const int32_t *places = static_cast<const int32_t *>(table(at, "place", T, k, at::kInt, dev));
    const Tensor out = a[4] == Py_None ? fresh(x, {T * k, D}, type) : tensor(a[4], "out", 2);
    const Matrix mo = any_rows(out, "out", T * k, D, type, dev);
    if (a[4] != Py_None) apart(out, "out", x, "x"), apart(out, "out", at, "place");
    const int rc = cocod_expert_rows(h, T, (int)k, D, m.data, m.ld, places, mo.data, mo.ld, type_code(type), current(dev));
    return rc == COCOD_OK && a[4] != Py_None ? given(a[4]) : code_or(rc, out);
}

// (handle, device, rows, place, weights or None, out or None, type)
PyObject *expert_join(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]);
    const Tensor &x = tensor(a[2], "rows", 2), &at = tensor(a[3], "place", 2);
    const int64_t T = at.size(0), k = at.size(1), D = x.size(1);
    const at::ScalarType type = value_type(x, "rows"), out_type = result_type(a[5], whole(a[6]), type);
    const Matrix m = any_rows(x, "rows", T * k, D, type, dev);
    const int32_t *places = static_cast<const int32_t *>(table(at, "place", T, k, at::kInt, dev));
    const float *w = a[4] == Py_None ? nullptr : static_cast<const float *>(table(tensor(a[4], "weights", 2), "weights", T, k, at::kFloat, dev));
    const Tensor out = a[5] == Py_None ? fresh(x, {T, D}, out_type) : tensor(a[5], "out", 2);
    const Matrix mo = any_rows(out, "out", T, D, out_type, dev);
    if (a[5] != Py_None) apart(out, "out", x, "rows"), apart(out, "out", at, "place"), apart(out, "out", a[4], "weights");
    const int rc = cocod_expert_join(h, T, (int)k, D, m.data, m.ld, type_code(type), places, w, mo.data, mo.ld, type_code(out_type), current(dev));
    return rc == COCOD_OK && a[5] != Py_None ? given(a[5]) : code_or(rc, out);
}

// (handle, device, dy, rows, place, weights, out or None): (the rows' gradient, the weights')
PyObject *expert_join_grad(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]);
    const Tensor &dy = tensor(a[2], "dy", 2), &x = tensor(a[3], "rows", 2), &at = tensor(a[4], "place", 2);
    const int64_t T = at.size(0), k = at.size(1), D = x.size(1);
    const at::ScalarType type = value_type(x, "rows");
    const Matrix md = any_rows(dy, "dy", T, D, type, dev), m = any_rows(x, "rows", T * k, D, type, dev);
    const int32_t *places = static_cast<const int32_t *>(table(at, "place", T, k, at::kInt, dev));
    const float *w = static_cast<const float *>(table(tensor(a[5], "weights", 2), "weights", T, k, at::kFloat, dev));
    const Tensor out = a[6] == Py_None ? fresh(x, {T * k, D}, type) : tensor(a[6], "out", 2), dw = fresh(x, {T, k}, at::kFloat);
    const Matrix mo = any_rows(out, "out", T * k, D, type, dev);
    if (a[6] != Py_None) apart(out, "out", dy, "dy"), apart(out, "out", x, "rows"), apart(out, "out", at, "place"), apart(out, "out", a[5], "weights");
    const int rc = cocod_expert_join_grad(h, T, (int)k, D, md.data, md.ld, m.data, m.ld, places, w, mo.data, mo.ld, static_cast<float *>(dw.data_ptr()),
                                          type_code(type), current(dev));
    if (rc != COCOD_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NN)", a[6] == Py_None ? THPVariable_Wrap(out) : given(a[6]), THPVariable_Wrap(dw));
}

// ------------------------------------------------------------------------------------------ log probabilities
inline float number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw std::runtime_error("");
    return (float)v;
}
int64_t alternatives(PyObject *o, int64_t V)
{
    const int64_t top = whole(o);
    if (top < 0 || top > COCOD_LM_MAX_TOP || top > V)
        throw std::invalid_argument("top: 0 to " + std::to_string(COCOD_LM_MAX_TOP) + " alternatives, at most as many as there are tokens; got " + std::to_string(top));
    return top;
}
const int32_t *given_tokens(PyObject *o, int64_t M, int64_t dev)
{
    return o == Py_None ? nullptr : static_cast<const int32_t *>(vector(tensor(o, "tokens", 1), "tokens", M, at::kInt, dev));
}

// (handle, device, logits, tokens or None, top, scale): (logp or None, entropy, log_sum, top_logp or None, top_tokens or None)
PyObject *token_logprobs(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]);
    const Tensor &x = tensor(a[2], "logits", 2);
    const int64_t M = x.size(0), V = x.size(1), top = alternatives(a[4], V);
    const at::ScalarType type = value_type(x, "logits");
    const Matrix m = any_rows(x, "logits", M, V, type, dev);
    const int32_t *tokens = given_tokens(a[3], M, dev);
    const float scale = number(a[5]);
    const int64_t padded = (M + 3) / 4 * 4, wide = (M * top + 3) / 4 * 4;          // (parts at multiples of 16 bytes)
    const Tensor all = fresh(x, {3 * padded + 2 * wide}, at::kFloat);
    float *p = static_cast<float *>(all.data_ptr());
    const int rc = cocod_token_logprobs(h, M, V, m.data, m.ld, type_code(type), tokens, scale, (int)top, p, p + padded, p + 2 * padded, p + 3 * padded,
                                        reinterpret_cast<int32_t *>(p + 3 * padded + wide), current(dev));
    if (rc != COCOD_OK) return PyLong_FromLong(rc);
    const auto part = [&](bool there, int64_t at, at::IntArrayRef shape, at::ScalarType kind) {
        return there ? THPVariable_Wrap(part_of(all, 4 * at, shape, kind)) : none();
    };
    return Py_BuildValue("(NNNNN)", part(a[3] != Py_None, 0, {M}, at::kFloat), part(true, padded, {M}, at::kFloat), part(true, 2 * padded, {M}, at::kFloat),
                         part(top > 0, 3 * padded, {M, top}, at::kFloat), part(top > 0, 3 * padded + wide, {M, top}, at::kInt));
}

// (handle, device, logits, tokens or None, scale, top_tokens or None, log_sum, entropy or None, d_logp or None, d_entropy or None, d_top or None,
// out or None)
PyObject *token_logprobs_grad(PyObject *const *a)
{
    cocod_lm_handle *h = handle(a[0]);
    const int64_t dev = device(a[1]);
    const Tensor &x = tensor(a[2], "logits", 2);
    const int64_t M = x.size(0), V = x.size(1);
    const at::ScalarType type = value_type(x, "logits");
    const Matrix m = any_rows(x, "logits", M, V, type, dev);
    const int32_t *tokens = given_tokens(a[3], M, dev);
    const float scale = number(a[4]);
    const auto row_values = [&](PyObject *o, const char *name) {
        return o == Py_None ? nullptr : static_cast<const float *>(vector(tensor(o, name, 1), name, M, at::kFloat, dev));
    };
    if (a[8] != Py_None && a[3] == Py_None) throw std::invalid_argument("d_logp: there are no tokens whose log probabilities it could belong to");
    if (a[9] != Py_None && a[7] == Py_None) throw std::invalid_argument("d_entropy: the entropy is needed");
    if (a[10] != Py_None && a[5] == Py_None) throw std::invalid_argument("d_top: the top tokens are needed");
    const float *log_sum = row_values(a[6], "log_sum"), *entropy = row_values(a[7], "entropy"), *d_logp = row_values(a[8], "d_logp"),
                *d_entropy = row_values(a[9], "d_entropy"), *d_top = nullptr;
    if (a[6] == Py_None) throw std::invalid_argument("log_sum: need a tensor");
    const int32_t *top_tokens = nullptr;
    int64_t top = 0;
    if (a[10] != Py_None) {
        const Tensor &t = tensor(a[5], "top_tokens", 2);
        top = t.size(1);
        if (top > COCOD_LM_MAX_TOP || top > V) refuse("top_tokens", "at most " + std::to_string(COCOD_LM_MAX_TOP) + " columns, and no more than tokens", t);
        top_tokens = static_cast<const int32_t *>(table(t, "top_tokens", M, top, at::kInt, dev));
        d_top = static_cast<const float *>(table(tensor(a[10], "d_top", 2), "d_top", M, top, at::kFloat, dev));
    }
    const Tensor out = a[11] == Py_None ? fresh(x, {M, V}, type) : tensor(a[11], "out", 2);
    const Matrix mo = any_rows(out, "out", M, V, type, dev);
    if (a[11] != Py_None) {
        apart(out, "out", x, "logits", true);
        apart(out, "out", a[3], "tokens");
        apart(out, "out", a[6], "log_sum");
        apart(out, "out", a[8], "d_logp");
        apart(out, "out", a[9], "d_entropy");
        apart(out, "out", a[10], "d_top");
        if (d_entropy != nullptr) apart(out, "out", a[7], "entropy");
        if (d_top != nullptr) apart(out, "out", a[5], "top_tokens");
    }
    const int rc = cocod_token_logprobs_grad(h, M, V, m.data, m.ld, type_code(type), tokens, scale, (int)top, top_tokens, log_sum, entropy, d_logp, d_entropy, d_top,
                                             mo.data, mo.ld, current(dev));
    return rc == COCOD_OK && a[11] != Py_None ? given(a[11]) : code_or(rc, out);
}

// ------------------------------------------------------------------------------------------ AdamW
// (handle, device, parameters, gradients, copies or None, gradients' factor or None): lists or tuples of the tensors the optimizer was made for, as many and
// of the same sizes (the kernels go by those); a gradient or a copy may be None
PyObject *adamw_step(PyObject *const *a)
{
    auto *h = reinterpret_cast<cocod_adamw_handle *>(handle(a[0]));
    const int64_t dev = device(a[1]);
    const bool copied = a[4] != Py_None;
    const auto sequence = [](PyObject *o) { return PyList_Check(o) || PyTuple_Check(o); };
    if (!sequence(a[2]) || !sequence(a[3]) || (copied && !sequence(a[4]))) throw std::invalid_argument("need lists of tensors");
    int n = 0;
    const int64_t *sizes = cocod_adamw_sizes(h, &n);
    if (PySequence_Fast_GET_SIZE(a[2]) != n) throw std::invalid_argument("params: need the " + std::to_string(n) + " that the optimizer was made for");
    if (PySequence_Fast_GET_SIZE(a[3]) != n || (copied && PySequence_Fast_GET_SIZE(a[4]) != n))
        throw std::invalid_argument("grads: need " + std::to_string(n) + ", one for each parameter (None: it stays as it is)");
    std::vector<void *> params(n), copies(copied ? n : 0);
    std::vector<const void *> grads(n);
    at::ScalarType types[2] = {at::kFloat, at::kFloat};
    bool first[2] = {true, true};
    const auto one = [&](PyObject *o, const char *name, int64_t size, int which) -> const Tensor & {
        const Tensor &t = tensor(o, name, -1);
        if (first[which]) types[which] = value_type(t, name), first[which] = false;
        if (!there(t, types[which], dev) || t.numel() != size || !t.is_contiguous())
            refuse(name, std::to_string(size) + " contiguous " + c10::toString(types[which]) + place(dev) + ", as the first one", t);
        return t;
    };
    for (int i = 0; i < n; ++i) {
        params[i] = one(PySequence_Fast_GET_ITEM(a[2], i), "params", sizes[i], 0).data_ptr();
        PyObject *g = PySequence_Fast_GET_ITEM(a[3], i), *c = copied ? PySequence_Fast_GET_ITEM(a[4], i) : Py_None;
        grads[i] = g == Py_None ? nullptr : one(g, "grads", sizes[i], 1).data_ptr();
        if (grads[i] != nullptr && grads[i] == params[i]) throw std::invalid_argument("grads: lies on its parameter");
        if (c == Py_None) continue;
        const Tensor &t = tensor(c, "copies", -1);
        if (!there(t, at::kBFloat16, dev) || t.numel() != sizes[i] || !t.is_contiguous()) refuse("copies", std::to_string(sizes[i]) + " contiguous BFloat16" + place(dev), t);
        copies[i] = t.data_ptr();
    }
    const float *factor = a[5] == Py_None ? nullptr : [&] {
        const Tensor &t = tensor(a[5], "grad_scale", -1);
        if (!there(t, at::kFloat, dev) || t.numel() != 1) refuse("grad_scale", "one Float" + place(dev), t);
        return static_cast<const float *>(t.data_ptr());
    }();
    const int rc = cocod_adamw_step(h, params.data(), type_code(types[0]), grads.data(), type_code(types[1]), copied ? copies.data() : nullptr, factor, current(dev));
    for (int i = 0; i < n && rc == COCOD_OK; ++i) {
        if (grads[i] == nullptr) continue;
        written(PySequence_Fast_GET_ITEM(a[2], i));
        if (copied && copies[i] != nullptr) written(PySequence_Fast_GET_ITEM(a[4], i));
    }
    return PyLong_FromLong(rc);
}

// (handle, device, values, a tensor of the state, stream or None: the current one): the moments in fp32
PyObject *adamw_moments(PyObject *const *a)
{
    auto *h = reinterpret_cast<cocod_adamw_handle *>(handle(a[0]));
    const int64_t dev = device(a[1]), values = whole(a[2]);
    const Tensor &like = tensor(a[3], "state", -1);
    const Tensor m = fresh(like, {values}, at::kFloat), v = fresh(like, {values}, at::kFloat);
    cocod_stream_t stream = a[4] == Py_None ? current(dev) : reinterpret_cast<cocod_stream_t>(whole(a[4]));
    const int rc = cocod_adamw_moments(h, static_cast<float *>(m.data_ptr()), static_cast<float *>(v.data_ptr()), stream);
    return rc == COCOD_OK ? Py_BuildValue("(NN)", THPVariable_Wrap(m), THPVariable_Wrap(v)) : PyLong_FromLong(rc);
}

#define METHOD(name, f, n) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<f, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    METHOD("grouped_forward", rows_product<true>, 7),
    METHOD("grouped_input_grad", rows_product<false>, 7),
    METHOD("grouped_weight_grad", weight_grad, 7),
    METHOD("grouped_weight_grad_packed", weight_grad_packed, 12),
    METHOD("act_pack_new", act_pack_new, 3),
    METHOD("act_pack_into", act_pack_into, 8),
    METHOD("act_unpack", act_unpack, 9),
    METHOD("act_relu_grad", act_relu_grad, 8),
    METHOD("vocab_loss", vocab<false>, 8),
    METHOD("vocab_loss_grad", vocab<true>, 10),
    METHOD("expert_sort", expert_sort, 4),
    METHOD("expert_rows", expert_rows, 5),
    METHOD("expert_join", expert_join, 7),
    METHOD("expert_join_grad", expert_join_grad, 7),
    METHOD("token_logprobs", token_logprobs, 6),
    METHOD("token_logprobs_grad", token_logprobs_grad, 12),
    METHOD("adamw_step", adamw_step, 6),
    METHOD("adamw_moments", adamw_moments, 5),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lm_binding", "Marshalling for the language-model operators (used by lm.py).", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lm_binding(void) { return PyModule_Create(&module); }

// What the native halves of the operators' calls share: arguments out of their Python objects, the stream that a call is queued on, and memory for what the
// caller has not given.
#pragma once
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/StreamGuard.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/adahop.h"

namespace {

// A refused argument: the Python exception is set, the call unwinds to HANDLE_TH_ERRORS.
[[noreturn]] inline void refuse(PyObject *type, const std::string &text)
{
    PyErr_SetString(type, text.c_str());
    throw python_error();
}

struct object_t { // one reference
    PyObject *p;
    explicit object_t(PyObject *o) : p(o)
    {
        if (!p) throw python_error();
    }
    ~object_t() { Py_XDECREF(p); }
    object_t(const object_t &) = delete;
    object_t &operator=(const object_t &) = delete;
    PyObject *release()
    {
        PyObject *const o = p;
        p = nullptr;
        return o;
    }
};

inline int64_t integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}

inline float number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return (float)v;
}

inline bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v != 0;
}

// What a call's tensors have to agree in.
struct frame_t {
    int64_t rows, cols;
    at::Device device;
};

inline const at::Tensor &tensor_of(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, std::string(what) + ": a tensor wanted, not " + Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}

inline std::string shape_of(const at::Tensor &t)
{
    std::string s = "[";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "]";
}

inline int f32_of(const at::Tensor &t, const char *what)
{
    if (t.scalar_type() != at::kBFloat16 && t.scalar_type() != at::kFloat) refuse(PyExc_TypeError, std::string(what) + ": bfloat16 or float32 wanted, not " + toString(t.scalar_type()));
    return t.scalar_type() == at::kFloat;
}

inline adahop_tensor_t matrix(PyObject *o, const frame_t &f, int64_t rows, const char *what)
{
    if (o == Py_None) return {};
    const at::Tensor &t = tensor_of(o, what);
    const int f32 = f32_of(t, what);
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != f.cols || (rows > 0 && f.cols > 1 && t.stride(1) != 1) || t.device() != f.device)
        refuse(PyExc_ValueError, std::string(what) + ": a [" + std::to_string(rows) + ", " + std::to_string(f.cols) + "] tensor with unit column stride on " + f.device.str() +
                                     " wanted, not " + shape_of(t) + " on " + t.device().str());
    return {t.data_ptr(), rows > 1 ? t.stride(0) : f.cols, f32};
}

inline adahop_tensor_t matrix(PyObject *o, const frame_t &f, const char *what) { return matrix(o, f, f.rows, what); }

inline adahop_tensor_t vector(PyObject *o, const frame_t &f, const char *what)
{
    if (o == Py_None) return {};
    const at::Tensor &t = tensor_of(o, what);
    const int f32 = f32_of(t, what);
    if (t.dim() != 1 || t.size(0) != f.cols || (f.cols > 1 && t.stride(0) != 1) || t.device() != f.device)
        refuse(PyExc_ValueError, std::string(what) + ": a dense vector of " + std::to_string(f.cols) + " elements on " + f.device.str() + " wanted, not " + shape_of(t) + " on " + t.device().str());
    return {t.data_ptr(), f.cols, f32};
}

inline float *floats(PyObject *o, int64_t n, const frame_t &f, const char *what)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor_of(o, what);
    if (t.scalar_type() != at::kFloat || t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1) || t.device() != f.device)
        refuse(PyExc_ValueError, std::string(what) + ": a dense float32 vector of " + std::to_string(n) + " elements on " + f.device.str() + " wanted");
    return static_cast<float *>(t.data_ptr());
}

inline adahop_ckpt8_t checkpoint(PyObject *o, const frame_t &f, const char *what)
{
    if (o == Py_None) return {};
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 2) refuse(PyExc_TypeError, std::string(what) + ": a pair (codes, scales) wanted");
    const int64_t width[2] = {f.cols, (f.cols + 31) / 32}, ld[2] = {(f.cols + 15) / 16 * 16, width[1]};
    uint8_t *p[2];
    int64_t stride[2];
    for (int i = 0; i < 2; ++i) {
        const at::Tensor &t = tensor_of(PyTuple_GET_ITEM(o, i), what);
        if (t.scalar_type() != at::kByte || t.dim() != 2 || t.size(0) != f.rows || t.size(1) != width[i] || (f.rows > 0 && width[i] > 1 && t.stride(1) != 1) || t.device() != f.device)
            refuse(PyExc_ValueError, std::string(what) + ": uint8 tensors [" + std::to_string(f.rows) + ", " + std::to_string(width[0]) + "] and [" + std::to_string(f.rows) + ", " +
                                         std::to_string(width[1]) + "] with unit column stride on " + f.device.str() + " wanted");
        p[i] = static_cast<uint8_t *>(t.data_ptr());
        stride[i] = f.rows > 1 ? t.stride(0) : ld[i];
    }
    return {p[0], p[1], stride[0], stride[1]};
}

inline bool is_checkpoint(PyObject *o) { return PyTuple_Check(o); }

// The frame of a call by the tensor whose shape the others have to have.
inline frame_t frame_of(PyObject *o, const char *what)
{
    const at::Tensor &t = tensor_of(o, what);
    if (t.dim() != 2) refuse(PyExc_ValueError, std::string(what) + ": two dimensions wanted, not " + shape_of(t));
    return {t.size(0), t.size(1), t.device()};
}

inline frame_t frame_of_checkpoint(PyObject *o, const char *what)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 2) refuse(PyExc_TypeError, std::string(what) + ": a pair (codes, scales) wanted");
    return frame_of(PyTuple_GET_ITEM(o, 0), what);
}

// ---- the stream, and outputs that the caller has not given --------------------------------------------------------------------
PyObject *current_stream = nullptr; // a callable: the handle of torch's current stream on the current device

inline void *handle_of(PyObject *o)
{
    const unsigned long long h = PyLong_AsUnsignedLongLongMask(o);
    if (h == (unsigned long long)-1 && PyErr_Occurred()) throw python_error();
    return reinterpret_cast<void *>((uintptr_t)h);
}

inline int64_t integer_attribute(PyObject *o, const char *name)
{
    const object_t v(PyObject_GetAttrString(o, name));
    return integer(v.p);
}

// Where a call's work is queued: on the tensors' device, on the stream that the caller names (a torch stream or a handle) or, None, on the current one.
//
// What a call allocates while it names another stream than the current one comes from that stream's memory, which its earlier work may still use and its
// later work alone gets back: an output that the caller drops at once, or a workspace, is nobody else's before the kernels are done with it.  The current stream is
// recorded on such outputs, so that one may be read there (once it has waited for the other) and dropped.  A bare handle has no memory of its own: with one of another
// stream all outputs and workspaces have to be the caller's.
class queue_t {
public:
    queue_t(PyObject *o, const frame_t &f) : device(f.device)
    {
        const bool torch_stream = o != Py_None && !PyIndex_Check(o);
        if (torch_stream && !PyObject_HasAttrString(o, "cuda_stream")) refuse(PyExc_TypeError, std::string("stream: a torch.cuda.Stream or a handle wanted, not ") + Py_TYPE(o)->tp_name);
        if (!device.is_cuda()) return; // refused by handle(), behind what else is wrong
        on.reset_device(device);
        if (torch_stream) {
            const c10::Stream s = c10::Stream::unpack3(integer_attribute(o, "stream_id"), (c10::DeviceIndex)integer_attribute(o, "device_index"), (c10::DeviceType)integer_attribute(o, "device_type"));
            if (s.device() != device) refuse(PyExc_ValueError, "stream: one of " + device.str() + " wanted, not of " + s.device().str());
            const c10::Stream now = c10::impl::VirtualGuardImpl(device.type()).getStream(device);
            if (s != now) {
                before = now;
                as.reset_stream(s);
            }
        }
        const object_t now(PyObject_CallNoArgs(current_stream));
        at = handle_of(now.p);
        if (o != Py_None && !torch_stream) {
            void *const given = handle_of(o);
            allocates = given == at;
            at = given;
        }
    }
    // The stream's, asked for when the arguments have been checked.  What the frame's tensors hold has to be where a kernel can read it.
    void *handle() const
    {
        if (!device.is_cuda()) refuse(PyExc_ValueError, "tensors on a GPU wanted, not on " + device.str());
        return at;
    }
    at::Tensor scratch(at::IntArrayRef shape, at::ScalarType type) const
    {
        if (!allocates) refuse(PyExc_ValueError, "a bare handle of another stream than the current one needs all outputs and workspaces given (or a torch.cuda.Stream)");
        return at::empty(shape, at::TensorOptions().dtype(type).device(device));
    }
    at::Tensor output(at::IntArrayRef shape, at::ScalarType type) const
    {
        at::Tensor t = scratch(shape, type);
        if (before) t.record_stream(*before);
        return t;
    }

    const at::Device device;

private:
    c10::OptionalDeviceGuard on;
    c10::OptionalStreamGuard as;
    std::optional<c10::Stream> before; // the current one, where the call is on another
    void *at = nullptr;
    bool allocates = true;
};

inline PyObject *empty(at::IntArrayRef shape, at::ScalarType type, const queue_t &q) { return THPVariable_Wrap(q.output(shape, type)); }

inline PyObject *empty_checkpoint(const frame_t &f, const queue_t &q)
{
    const int64_t ld = (f.cols + 15) / 16 * 16;
    at::Tensor codes = q.output({f.rows, ld}, at::kByte);
    if (ld != f.cols) codes = codes.narrow(1, 0, f.cols);
    const object_t c(THPVariable_Wrap(codes)), s(empty({f.rows, (f.cols + 31) / 32}, at::kByte, q));
    return PyTuple_Pack(2, c.p, s.p);
}

// The object itself, or a new one of what make() says: one reference either way.
template <class F> inline PyObject *given_or(PyObject *o, F make)
{
    if (o == Py_None) return make();
    Py_INCREF(o);
    return o;
}

inline PyObject *none()
{
    Py_INCREF(Py_None);
    return Py_None;
}

inline at::ScalarType type_of(PyObject *o) { return THPVariable_Unpack(o).scalar_type(); }

// A workspace of so many bytes: the caller's, or a new one (released when the call returns, to its stream's later work).
struct workspace_t {
    at::Tensor own;
    void *data = nullptr;
    size_t bytes = 0;
    workspace_t(PyObject *o, size_t need, const queue_t &q)
    {
        if (o == Py_None) {
            if (!need) return;
            own = q.scratch({(int64_t)need}, at::kByte);
        } else {
            own = tensor_of(o, "workspace");
            if (own.scalar_type() != at::kByte || own.dim() != 1 || (own.size(0) > 1 && own.stride(0) != 1) || own.device() != q.device)
                refuse(PyExc_ValueError, "workspace: a dense uint8 vector on " + q.device.str() + " wanted");
        }
        data = own.data_ptr();
        bytes = (size_t)own.numel();
    }
};

// (status, dict) of the names' objects, whose references go into it.
inline PyObject *answer(int status, std::initializer_list<std::pair<PyObject *, PyObject *>> items)
{
    const object_t d(PyDict_New()), s(PyLong_FromLong(status));
    for (const auto &i : items)
        if (PyDict_SetItem(d.p, i.first, i.second) < 0) throw python_error();
    return PyTuple_Pack(2, s.p, d.p);
}

inline PyObject *answer(int status, PyObject *one)
{
    const object_t s(PyLong_FromLong(status));
    return PyTuple_Pack(2, s.p, one);
}

inline void expect(Py_ssize_t n, Py_ssize_t wanted)
{
    if (n != wanted) refuse(PyExc_TypeError, "wrong number of arguments");
}

} // namespace

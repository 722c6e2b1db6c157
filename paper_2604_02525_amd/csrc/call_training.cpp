// The host side of the training operators' calls: arguments out of their Python objects, checked against each other, missing outputs
// allocated, the C entry point.  Through ctypes and torch's Python functions the call of the block norm took 11.9 us, its backward 30, while their kernels take
// 4 to 6 on a few rows; here the two calls take 5.4 and 7.6 us, their launches among them.
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

struct entries_t {
    decltype(&adahop_ckpt8_pack) pack;
    decltype(&adahop_ckpt8_unpack) unpack;
    decltype(&adahop_swiglu) swiglu;
    decltype(&adahop_swiglu_backward) swiglu_backward;
    decltype(&adahop_block_norm) norm;
    decltype(&adahop_block_norm_backward) norm_backward;
    decltype(&adahop_block_norm_backward_workspace_bytes) norm_backward_bytes;
    decltype(&adahop_ckpt8_wgrad) wgrad;
    decltype(&adahop_ckpt8_wgrad_workspace_bytes) wgrad_bytes;
} entry;

// A refused argument: the Python exception is set, the call unwinds to HANDLE_TH_ERRORS.
[[noreturn]] void refuse(PyObject *type, const std::string &text)
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

int64_t integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}

float number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return (float)v;
}

bool truth(PyObject *o)
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

const at::Tensor &tensor_of(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, std::string(what) + ": a tensor wanted, not " + Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}

std::string shape_of(const at::Tensor &t)
{
    std::string s = "[";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "]";
}

int f32_of(const at::Tensor &t, const char *what)
{
    if (t.scalar_type() != at::kBFloat16 && t.scalar_type() != at::kFloat) refuse(PyExc_TypeError, std::string(what) + ": bfloat16 or float32 wanted, not " + toString(t.scalar_type()));
    return t.scalar_type() == at::kFloat;
}

adahop_tensor_t matrix(PyObject *o, const frame_t &f, int64_t rows, const char *what)
{
    if (o == Py_None) return {};
    const at::Tensor &t = tensor_of(o, what);
    const int f32 = f32_of(t, what);
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != f.cols || (rows > 0 && f.cols > 1 && t.stride(1) != 1) || t.device() != f.device)
        refuse(PyExc_ValueError, std::string(what) + ": a [" + std::to_string(rows) + ", " + std::to_string(f.cols) + "] tensor with unit column stride on " + f.device.str() +
                                     " wanted, not " + shape_of(t) + " on " + t.device().str());
    return {t.data_ptr(), rows > 1 ? t.stride(0) : f.cols, f32};
}

adahop_tensor_t matrix(PyObject *o, const frame_t &f, const char *what) { return matrix(o, f, f.rows, what); }

adahop_tensor_t vector(PyObject *o, const frame_t &f, const char *what)
{
    if (o == Py_None) return {};
    const at::Tensor &t = tensor_of(o, what);
    const int f32 = f32_of(t, what);
    if (t.dim() != 1 || t.size(0) != f.cols || (f.cols > 1 && t.stride(0) != 1) || t.device() != f.device)
        refuse(PyExc_ValueError, std::string(what) + ": a dense vector of " + std::to_string(f.cols) + " elements on " + f.device.str() + " wanted, not " + shape_of(t) + " on " + t.device().str());
    return {t.data_ptr(), f.cols, f32};
}

float *floats(PyObject *o, int64_t n, const frame_t &f, const char *what)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor_of(o, what);
    if (t.scalar_type() != at::kFloat || t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1) || t.device() != f.device)
        refuse(PyExc_ValueError, std::string(what) + ": a dense float32 vector of " + std::to_string(n) + " elements on " + f.device.str() + " wanted");
    return static_cast<float *>(t.data_ptr());
}

adahop_ckpt8_t checkpoint(PyObject *o, const frame_t &f, const char *what)
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

bool is_checkpoint(PyObject *o) { return PyTuple_Check(o); }

// The frame of a call by the tensor whose shape the others have to have.
frame_t frame_of(PyObject *o, const char *what)
{
    const at::Tensor &t = tensor_of(o, what);
    if (t.dim() != 2) refuse(PyExc_ValueError, std::string(what) + ": two dimensions wanted, not " + shape_of(t));
    return {t.size(0), t.size(1), t.device()};
}

frame_t frame_of_checkpoint(PyObject *o, const char *what)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 2) refuse(PyExc_TypeError, std::string(what) + ": a pair (codes, scales) wanted");
    return frame_of(PyTuple_GET_ITEM(o, 0), what);
}

// ---- the stream, and outputs that the caller has not given --------------------------------------------------------------------
PyObject *current_stream = nullptr; // a callable: the handle of torch's current stream on the current device

void *handle_of(PyObject *o)
{
    const unsigned long long h = PyLong_AsUnsignedLongLongMask(o);
    if (h == (unsigned long long)-1 && PyErr_Occurred()) throw python_error();
    return reinterpret_cast<void *>((uintptr_t)h);
}

int64_t integer_attribute(PyObject *o, const char *name)
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

PyObject *empty(at::IntArrayRef shape, at::ScalarType type, const queue_t &q) { return THPVariable_Wrap(q.output(shape, type)); }

PyObject *empty_checkpoint(const frame_t &f, const queue_t &q)
{
    const int64_t ld = (f.cols + 15) / 16 * 16;
    at::Tensor codes = q.output({f.rows, ld}, at::kByte);
    if (ld != f.cols) codes = codes.narrow(1, 0, f.cols);
    const object_t c(THPVariable_Wrap(codes)), s(empty({f.rows, (f.cols + 31) / 32}, at::kByte, q));
    return PyTuple_Pack(2, c.p, s.p);
}

// The object itself, or a new one of what make() says: one reference either way.
template <class F> PyObject *given_or(PyObject *o, F make)
{
    if (o == Py_None) return make();
    Py_INCREF(o);
    return o;
}

PyObject *none()
{
    Py_INCREF(Py_None);
    return Py_None;
}

at::ScalarType type_of(PyObject *o) { return THPVariable_Unpack(o).scalar_type(); }

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

struct names_t {
    PyObject *a, *ckpt_g, *ckpt_u, *d_g, *d_u, *s, *h, *rstd_post, *rstd_pre, *ckpt_y, *ckpt_s, *d_x, *d_y, *d_w_post, *d_w_pre, *d_gate;
} name;

// (status, dict) of the names' objects, whose references go into it.
PyObject *answer(int status, std::initializer_list<std::pair<PyObject *, PyObject *>> items)
{
    const object_t d(PyDict_New()), s(PyLong_FromLong(status));
    for (const auto &i : items)
        if (PyDict_SetItem(d.p, i.first, i.second) < 0) throw python_error();
    return PyTuple_Pack(2, s.p, d.p);
}

PyObject *answer(int status, PyObject *one)
{
    const object_t s(PyLong_FromLong(status));
    return PyTuple_Pack(2, s.p, one);
}

void expect(Py_ssize_t n, Py_ssize_t wanted)
{
    if (n != wanted) refuse(PyExc_TypeError, "wrong number of arguments");
}

// The entry points are called with the interpreter's lock held: they queue work and return.

// pack(x, out, stream)
PyObject *pack(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 3);
    const frame_t f = frame_of(v[0], "x");
    const queue_t q(v[2], f);
    const adahop_tensor_t x = matrix(v[0], f, "x");
    const object_t out(given_or(v[1], [&] { return empty_checkpoint(f, q); }));
    const adahop_ckpt8_t k = checkpoint(out.p, f, "out");
    return answer(entry.pack(f.rows, f.cols, &x, &k, q.handle()), out.p);
    END_HANDLE_TH_ERRORS
}

// unpack(x8, col_scale, out, f32, stream)
PyObject *unpack(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 5);
    const frame_t f = frame_of_checkpoint(v[0], "x8");
    const queue_t q(v[4], f);
    const adahop_ckpt8_t x = checkpoint(v[0], f, "x8");
    const adahop_tensor_t scale = vector(v[1], f, "col_scale");
    const object_t out(given_or(v[2], [&] { return empty({f.rows, f.cols}, truth(v[3]) ? at::kFloat : at::kBFloat16, q); }));
    const adahop_tensor_t o = matrix(out.p, f, "out");
    return answer(entry.unpack(f.rows, f.cols, &x, &scale, &o, q.handle()), out.p);
    END_HANDLE_TH_ERRORS
}

// swiglu(g, u, a, ckpt_g, ckpt_u, keep8, stream)
PyObject *swiglu(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 7);
    const frame_t f = frame_of(v[0], "g");
    const queue_t q(v[6], f);
    const bool keep = truth(v[5]);
    adahop_swiglu_t p = {};
    p.rows = f.rows, p.cols = f.cols;
    p.g = matrix(v[0], f, "g"), p.u = matrix(v[1], f, "u");
    const object_t a(given_or(v[2], [&] { return empty({f.rows, f.cols}, at::kBFloat16, q); }));
    const object_t kg(given_or(v[3], [&] { return keep ? empty_checkpoint(f, q) : none(); })), ku(given_or(v[4], [&] { return keep ? empty_checkpoint(f, q) : none(); }));
    p.a = matrix(a.p, f, "a"), p.ckpt_g = checkpoint(kg.p, f, "ckpt_g"), p.ckpt_u = checkpoint(ku.p, f, "ckpt_u");
    return answer(entry.swiglu(&p, q.handle()), {{name.a, a.p}, {name.ckpt_g, kg.p}, {name.ckpt_u, ku.p}});
    END_HANDLE_TH_ERRORS
}

// swiglu_backward(g, u, d_a, d_g, d_u, a, stream)
PyObject *swiglu_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 7);
    const frame_t f = frame_of(v[2], "d_a");
    const queue_t q(v[6], f);
    adahop_swiglu_t p = {};
    p.rows = f.rows, p.cols = f.cols;
    if (is_checkpoint(v[0]))
        p.ckpt_g = checkpoint(v[0], f, "g");
    else
        p.g = matrix(v[0], f, "g");
    if (is_checkpoint(v[1]))
        p.ckpt_u = checkpoint(v[1], f, "u");
    else
        p.u = matrix(v[1], f, "u");
    if (is_checkpoint(v[5]))
        p.ckpt_a = checkpoint(v[5], f, "a");
    else
        p.a = matrix(v[5], f, "a");
    at::Tensor both;
    if (v[3] == Py_None && v[4] == Py_None) both = q.output({f.rows, 2 * f.cols}, at::kBFloat16);
    const auto half = [&](int64_t from) { return both.defined() ? THPVariable_Wrap(both.narrow(1, from, f.cols)) : empty({f.rows, f.cols}, at::kBFloat16, q); };
    const object_t dg(given_or(v[3], [&] { return half(0); })), du(given_or(v[4], [&] { return half(f.cols); }));
    p.d_a = matrix(v[2], f, "d_a"), p.d_g = matrix(dg.p, f, "d_g"), p.d_u = matrix(du.p, f, "d_u");
    return answer(entry.swiglu_backward(&p, q.handle()), {{name.d_g, dg.p}, {name.d_u, du.p}, {name.a, v[5]}});
    END_HANDLE_TH_ERRORS
}

// gate: None, a vector for all rows, or [gates, cols], each for gate_rows rows
void set_gate(adahop_block_norm_t &p, PyObject *gate, PyObject *gate_rows, const frame_t &f)
{
    if (gate == Py_None) return;
    if (tensor_of(gate, "gate").dim() == 1) {
        p.gate = vector(gate, f, "gate");
        p.gates = 1;
        p.gate_rows = f.rows > 1 ? f.rows : 1;
    } else {
        p.gates = THPVariable_Unpack(gate).dim() == 2 ? THPVariable_Unpack(gate).size(0) : -1;
        p.gate = matrix(gate, f, p.gates, "gate");
        p.gate_rows = integer(gate_rows);
    }
}

// block_norm(x, y, w_post, w_pre, gate, gate_rows, residual_scale, branch_scale, eps, post_norm, pre_norm, s, h, rstd_post, rstd_pre, ckpt_y, ckpt_s,
// stats, ckpt8, stream)
PyObject *block_norm(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 20);
    PyObject *const x = v[0], *const y = v[1];
    const frame_t f = frame_of(x == Py_None ? y : x, x == Py_None ? "y" : "x");
    const queue_t q(v[19], f);
    adahop_block_norm_t p = {};
    p.rows = f.rows, p.cols = f.cols;
    p.residual_scale = number(v[6]), p.branch_scale = number(v[7]), p.eps = number(v[8]);
    const bool has_y = y != Py_None, post = truth(v[9]) && has_y, pre = truth(v[10]), stats = truth(v[17]), keep = truth(v[18]);
    p.post_norm = post;
    p.x = matrix(x, f, "x"), p.y = matrix(y, f, "y"), p.w_post = vector(v[2], f, "w_post"), p.w_pre = vector(v[3], f, "w_pre");
    set_gate(p, v[4], v[5], f);
    const bool same = !has_y && p.residual_scale == 1.0f && (v[11] == Py_None || v[11] == x); // s = x is there already
    const auto vec = [&](bool wanted) { return wanted ? empty({f.rows}, at::kFloat, q) : none(); };
    const auto kept = [&](bool wanted) { return wanted ? empty_checkpoint(f, q) : none(); };
    const object_t s(same ? given_or(x, none) : given_or(v[11], [&] { return empty({f.rows, f.cols}, type_of(x == Py_None ? y : x), q); }));
    const object_t h(pre ? given_or(v[12], [&] { return empty({f.rows, f.cols}, at::kBFloat16, q); }) : none());
    const object_t r_post(given_or(v[13], [&] { return vec((stats || keep) && post); })), r_pre(given_or(v[14], [&] { return vec((stats || keep) && pre); }));
    const object_t ky(given_or(v[15], [&] { return kept(keep && has_y); })), ks(given_or(v[16], [&] { return kept(keep && pre); }));
    if (!same) p.s = matrix(s.p, f, "s");
    p.h = matrix(h.p, f, "h");
    p.rstd_post = floats(r_post.p, f.rows, f, "rstd_post"), p.rstd_pre = floats(r_pre.p, f.rows, f, "rstd_pre");
    p.ckpt_y = checkpoint(ky.p, f, "ckpt_y"), p.ckpt_s = checkpoint(ks.p, f, "ckpt_s");
    return answer(entry.norm(&p, q.handle()), {{name.s, s.p}, {name.h, h.p}, {name.rstd_post, r_post.p}, {name.rstd_pre, r_pre.p}, {name.ckpt_y, ky.p}, {name.ckpt_s, ks.p}});
    END_HANDLE_TH_ERRORS
}

// block_norm_backward(d_s, d_h, s, y, rstd_pre, rstd_post, w_post, w_pre, gate, gate_rows, residual_scale, branch_scale, post_norm, d_x, d_y, d_w_post,
// d_w_pre, d_gate, workspace, stream)
PyObject *block_norm_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 20);
    PyObject *const d_s = v[0], *const d_h = v[1], *const s = v[2], *const y = v[3];
    const bool has_s = d_s != Py_None, has_h = d_h != Py_None, has_y = y != Py_None;
    const frame_t f = frame_of(has_s ? d_s : d_h, has_s ? "d_s" : "d_h");
    const queue_t q(v[19], f);
    adahop_block_norm_t p = {};
    p.rows = f.rows, p.cols = f.cols;
    p.post_norm = truth(v[12]) && has_y;
    p.residual_scale = number(v[10]), p.branch_scale = number(v[11]);
    p.w_post = vector(v[6], f, "w_post"), p.w_pre = vector(v[7], f, "w_pre");
    set_gate(p, v[8], v[9], f);
    if (is_checkpoint(s))
        p.ckpt_s = checkpoint(s, f, "s");
    else
        p.s = matrix(s, f, "s");
    if (is_checkpoint(y))
        p.ckpt_y = checkpoint(y, f, "y");
    else
        p.y = matrix(y, f, "y");
    p.rstd_pre = floats(v[4], f.rows, f, "rstd_pre"), p.rstd_post = floats(v[5], f.rows, f, "rstd_post");
    p.d_s = matrix(d_s, f, "d_s"), p.d_h = matrix(d_h, f, "d_h");
    const auto like = [&](at::ScalarType type) { return empty({f.rows, f.cols}, type, q); };
    const auto vec = [&](bool wanted) { return wanted ? empty({f.cols}, at::kFloat, q) : none(); };
    const object_t dx(given_or(v[13], [&] { return like(has_s ? type_of(d_s) : p.s.data ? type_of(s) : type_of(d_h)); }));
    const object_t dy(given_or(v[14], [&] { return !has_y ? none() : like(has_h ? type_of(d_h) : p.y.data ? type_of(y) : at::kBFloat16); }));
    const object_t dwpost(given_or(v[15], [&] { return vec(v[6] != Py_None && has_y); })), dwpre(given_or(v[16], [&] { return vec(v[7] != Py_None && has_h); }));
    const object_t dgate(given_or(v[17], [&] { return v[8] == Py_None ? none() : empty(THPVariable_Unpack(v[8]).sizes(), type_of(v[8]), q); }));
    p.d_x = matrix(dx.p, f, "d_x"), p.d_y = matrix(dy.p, f, "d_y");
    p.d_w_post = floats(dwpost.p, f.cols, f, "d_w_post"), p.d_w_pre = floats(dwpre.p, f.cols, f, "d_w_pre");
    if (dgate.p != Py_None) p.d_gate = tensor_of(dgate.p, "d_gate").dim() == 1 ? vector(dgate.p, f, "d_gate") : matrix(dgate.p, f, p.gates, "d_gate");
    const workspace_t ws(v[18], entry.norm_backward_bytes(f.rows, f.cols, p.gate.data ? p.gate_rows : 0), q);
    return answer(entry.norm_backward(&p, ws.data, ws.bytes, q.handle()),
                  {{name.d_x, dx.p}, {name.d_y, dy.p}, {name.d_w_post, dwpost.p}, {name.d_w_pre, dwpre.p}, {name.d_gate, dgate.p}});
    END_HANDLE_TH_ERRORS
}

// wgrad(G, x8, col_scale, add, Cout, bf16, workspace, stream)
PyObject *wgrad(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 8);
    const frame_t g = frame_of(v[0], "G"), x = {g.rows, frame_of_checkpoint(v[1], "x8").cols, g.device}, c = {g.cols, x.cols, g.device};
    const queue_t q(v[7], g);
    adahop_tensor_t G = matrix(v[0], g, "G");
    if (g.rows <= 1) G.ld = (g.cols + 7) / 8 * 8;
    const adahop_ckpt8_t k = checkpoint(v[1], x, "x8");
    const adahop_tensor_t scale = vector(v[2], c, "col_scale"), add = matrix(v[3], c, "add");
    const object_t out(given_or(v[4], [&] { return empty({c.rows, c.cols}, truth(v[5]) ? at::kBFloat16 : at::kFloat, q); }));
    const adahop_tensor_t C = matrix(out.p, c, "Cout");
    const workspace_t ws(v[6], entry.wgrad_bytes(g.rows, g.cols, x.cols), q);
    return answer(entry.wgrad(g.rows, g.cols, x.cols, &G, &k, &scale, &add, &C, ws.data, ws.bytes, q.handle()), out.p);
    END_HANDLE_TH_ERRORS
}

// init_training(current_stream, addresses of the entry points, in the order of entries_t)
PyObject *init_training(PyObject *, PyObject *args)
{
    unsigned long long a[9];
    PyObject *stream;
    if (!PyArg_ParseTuple(args, "OKKKKKKKKK", &stream, a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7, a + 8)) return nullptr;
    Py_INCREF(stream); // (for the life of the process)
    current_stream = stream;
    entry = {reinterpret_cast<decltype(entry.pack)>(a[0]), reinterpret_cast<decltype(entry.unpack)>(a[1]), reinterpret_cast<decltype(entry.swiglu)>(a[2]),
             reinterpret_cast<decltype(entry.swiglu_backward)>(a[3]), reinterpret_cast<decltype(entry.norm)>(a[4]), reinterpret_cast<decltype(entry.norm_backward)>(a[5]),
             reinterpret_cast<decltype(entry.norm_backward_bytes)>(a[6]), reinterpret_cast<decltype(entry.wgrad)>(a[7]), reinterpret_cast<decltype(entry.wgrad_bytes)>(a[8])};
    Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"init_training", init_training, METH_VARARGS, nullptr}, FAST(pack), FAST(unpack), FAST(swiglu), FAST(swiglu_backward), FAST(block_norm),
                         FAST(block_norm_backward), FAST(wgrad), {nullptr, nullptr, 0, nullptr}};

} // namespace

// Adds the functions above to the binding's native module.
int add_training_calls(PyObject *module)
{
    PyObject **const to[] = {&name.a, &name.ckpt_g, &name.ckpt_u, &name.d_g, &name.d_u, &name.s, &name.h, &name.rstd_post, &name.rstd_pre, &name.ckpt_y, &name.ckpt_s,
                             &name.d_x, &name.d_y, &name.d_w_post, &name.d_w_pre, &name.d_gate};
    const char *const text[] = {"a", "ckpt_g", "ckpt_u", "d_g", "d_u", "s", "h", "rstd_post", "rstd_pre", "ckpt_y", "ckpt_s", "d_x", "d_y", "d_w_post", "d_w_pre", "d_gate"};
    for (size_t i = 0; i < sizeof to / sizeof *to; ++i)
        if (!(*to[i] = PyUnicode_InternFromString(text[i]))) return -1;
    return PyModule_AddFunctions(module, methods);
}

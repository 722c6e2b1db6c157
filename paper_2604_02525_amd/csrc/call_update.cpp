// The host side of the calls behind the last block (the loss over a vocabulary, orthogonalised updates), as call_training.cpp is for those around the products.
#include "call_common.h"

namespace {

struct entries_t {
    decltype(&adahop_linear_ce) ce;
    decltype(&adahop_linear_ce_backward) ce_backward;
    decltype(&adahop_linear_ce_workspace_bytes) ce_bytes;
    decltype(&adahop_orthogonalize) orthogonalize;
    decltype(&adahop_muon_update) muon;
    decltype(&adahop_newton_schulz_workspace_bytes) newton_schulz_bytes;
} entry;

struct names_t {
    PyObject *loss, *lse, *d_h, *d_w, *w, *momentum, *w_bf16;
} name;

const int64_t *targets_of(PyObject *o, const frame_t &f)
{
    const at::Tensor &t = tensor_of(o, "targets");
    if (t.scalar_type() != at::kLong) refuse(PyExc_TypeError, std::string("targets: int64 wanted, not ") + toString(t.scalar_type()));
    if (t.dim() != 1 || t.size(0) != f.rows || (f.rows > 1 && t.stride(0) != 1) || t.device() != f.device)
        refuse(PyExc_ValueError, "targets: a dense vector of " + std::to_string(f.rows) + " elements on " + f.device.str() + " wanted, not " + shape_of(t) + " on " + t.device().str());
    return static_cast<const int64_t *>(t.data_ptr());
}

// Both directions' operands: h [tokens, dim], w [vocab, dim].
frame_t operands(adahop_linear_ce_t &p, PyObject *h, PyObject *w, PyObject *targets, PyObject *logit_scale, PyObject *z_loss)
{
    const frame_t f = frame_of(h, "h"), v = {frame_of(w, "w").rows, f.cols, f.device};
    p.tokens = f.rows, p.dim = f.cols, p.vocab = v.rows;
    p.h = matrix(h, f, "h"), p.w = matrix(w, v, "w");
    if (p.h.f32 || p.w.f32) refuse(PyExc_TypeError, "h and w: bfloat16 wanted");
    // one row's stride says nothing: as rows of whole pieces would lie
    if (f.rows <= 1) p.h.ld = (f.cols + 7) / 8 * 8;
    if (v.rows <= 1) p.w.ld = (f.cols + 7) / 8 * 8;
    p.targets = targets_of(targets, f);
    p.logit_scale = number(logit_scale), p.z_loss = number(z_loss);
    return f;
}

// linear_ce(h, w, targets, logit_scale, z_loss, loss, lse, workspace, stream)
PyObject *linear_ce(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 9);
    const frame_t first = frame_of(v[0], "h");
    const queue_t q(v[8], first);
    adahop_linear_ce_t p = {};
    const frame_t f = operands(p, v[0], v[1], v[2], v[3], v[4]);
    const auto vec = [&] { return empty({f.rows}, at::kFloat, q); };
    const object_t loss(given_or(v[5], vec)), lse(given_or(v[6], vec));
    p.loss = floats(loss.p, f.rows, f, "loss"), p.lse = floats(lse.p, f.rows, f, "lse");
    const workspace_t ws(v[7], entry.ce_bytes(&p, 0), q);
    return answer(entry.ce(&p, ws.data, ws.bytes, q.handle()), {{name.loss, loss.p}, {name.lse, lse.p}});
    END_HANDLE_TH_ERRORS
}

// linear_ce_backward(h, w, targets, lse, d_loss, logit_scale, z_loss, d_h, d_w, add, want_h, want_w, d_w_bf16, workspace, stream)
PyObject *linear_ce_backward(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 15);
    const frame_t first = frame_of(v[0], "h");
    const queue_t q(v[14], first);
    adahop_linear_ce_t p = {};
    const frame_t f = operands(p, v[0], v[1], v[2], v[5], v[6]), c = {p.vocab, f.cols, f.device};
    if (v[3] == Py_None) refuse(PyExc_TypeError, "lse: a tensor wanted, not NoneType");
    p.lse = floats(v[3], f.rows, f, "lse");
    if (v[4] != Py_None) { // one number for all tokens may be an expanded one
        const at::Tensor &t = tensor_of(v[4], "d_loss");
        if (t.scalar_type() != at::kFloat || t.dim() != 1 || t.size(0) != f.rows || (f.rows > 1 && t.stride(0) != 1 && t.stride(0) != 0) || t.device() != f.device)
            refuse(PyExc_ValueError, "d_loss: a float32 vector of " + std::to_string(f.rows) + " elements, dense or expanded from one, on " + f.device.str() + " wanted");
        p.d_loss = static_cast<const float *>(t.data_ptr());
        p.d_loss_stride = f.rows > 1 ? t.stride(0) : 1;
    }
    const bool want_h = truth(v[10]), want_w = truth(v[11]);
    if ((!want_h && v[7] != Py_None) || (!want_w && (v[8] != Py_None || v[9] != Py_None))) refuse(PyExc_ValueError, "d_h, d_w, add: given for a gradient that is not wanted");
    const object_t dh(want_h ? given_or(v[7], [&] { return empty({f.rows, f.cols}, at::kBFloat16, q); }) : none());
    const object_t dw(want_w ? given_or(v[8], [&] { return empty({c.rows, c.cols}, truth(v[12]) ? at::kBFloat16 : at::kFloat, q); }) : none());
    p.d_h = matrix(dh.p, f, "d_h"), p.d_w = matrix(dw.p, c, "d_w"), p.add = matrix(v[9], c, "add");
    const workspace_t ws(v[13], entry.ce_bytes(&p, 1), q);
    return answer(entry.ce_backward(&p, ws.data, ws.bytes, q.handle()), {{name.d_h, dh.p}, {name.d_w, dw.p}});
    END_HANDLE_TH_ERRORS
}

int small_integer(PyObject *o, const char *what)
{
    const int64_t v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) refuse(PyExc_ValueError, std::string(what) + ": " + std::to_string(v) + " is out of range");
    return (int)v;
}

// steps, a, b, c, eps, scale
adahop_newton_schulz_t method_of(const frame_t &f, PyObject *const *v)
{
    return {f.rows, f.cols, small_integer(v[0], "steps"), number(v[1]), number(v[2]), number(v[3]), number(v[4]), number(v[5])};
}

// orthogonalize(g, out, f32, steps, a, b, c, eps, scale, workspace, stream)
PyObject *orthogonalize(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 11);
    const frame_t f = frame_of(v[0], "g");
    const queue_t q(v[10], f);
    const adahop_newton_schulz_t m = method_of(f, v + 3);
    const adahop_tensor_t g = matrix(v[0], f, "g");
    const object_t out(given_or(v[1], [&] { return empty({f.rows, f.cols}, truth(v[2]) ? at::kFloat : at::kBFloat16, q); }));
    const adahop_tensor_t o = matrix(out.p, f, "out");
    const workspace_t ws(v[9], entry.newton_schulz_bytes(f.rows, f.cols), q);
    return answer(entry.orthogonalize(&m, &g, &o, ws.data, ws.bytes, q.handle()), out.p);
    END_HANDLE_TH_ERRORS
}

// muon_update(w, g, momentum, rate, mu, weight_decay, nesterov, w_out, momentum_out, w_bf16, steps, a, b, c, eps, scale, workspace, stream)
PyObject *muon_update(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    expect(n, 18);
    const frame_t f = frame_of(v[0], "w");
    const queue_t q(v[17], f);
    const adahop_newton_schulz_t m = method_of(f, v + 10);
    tensor_of(v[1], "g"), tensor_of(v[2], "momentum");
    PyObject *const w_out = v[7] == Py_None ? v[0] : v[7], *const m_out = v[8] == Py_None ? v[2] : v[8];
    adahop_muon_t p = {};
    p.rows = f.rows, p.cols = f.cols;
    p.w = matrix(v[0], f, "w"), p.g = matrix(v[1], f, "g"), p.momentum = matrix(v[2], f, "momentum");
    p.w_out = matrix(w_out, f, "w_out"), p.momentum_out = matrix(m_out, f, "momentum_out"), p.w_bf16 = matrix(v[9], f, "w_bf16");
    p.rate = number(v[3]), p.mu = number(v[4]), p.weight_decay = number(v[5]);
    p.nesterov = truth(v[6]);
    const workspace_t ws(v[16], entry.newton_schulz_bytes(f.rows, f.cols), q);
    return answer(entry.muon(&m, &p, ws.data, ws.bytes, q.handle()), {{name.w, w_out}, {name.momentum, m_out}, {name.w_bf16, v[9]}});
    END_HANDLE_TH_ERRORS
}

// init_update(current_stream, addresses of the entry points, in the order of entries_t)
PyObject *init_update(PyObject *, PyObject *args)
{
    unsigned long long a[6];
    PyObject *stream;
    if (!PyArg_ParseTuple(args, "OKKKKKK", &stream, a, a + 1, a + 2, a + 3, a + 4, a + 5)) return nullptr;
    Py_INCREF(stream); // (for the life of the process)
    current_stream = stream;
    entry = {reinterpret_cast<decltype(entry.ce)>(a[0]), reinterpret_cast<decltype(entry.ce_backward)>(a[1]), reinterpret_cast<decltype(entry.ce_bytes)>(a[2]),
             reinterpret_cast<decltype(entry.orthogonalize)>(a[3]), reinterpret_cast<decltype(entry.muon)>(a[4]), reinterpret_cast<decltype(entry.newton_schulz_bytes)>(a[5])};
    Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"init_update", init_update, METH_VARARGS, nullptr}, FAST(linear_ce), FAST(linear_ce_backward), FAST(orthogonalize), FAST(muon_update),
                         {nullptr, nullptr, 0, nullptr}};

} // namespace

// Adds the functions above to the binding's native module.
int add_update_calls(PyObject *module)
{
    PyObject **const to[] = {&name.loss, &name.lse, &name.d_h, &name.d_w, &name.w, &name.momentum, &name.w_bf16};
    const char *const text[] = {"loss", "lse", "d_h", "d_w", "w", "momentum", "w_bf16"};
    for (size_t i = 0; i < sizeof to / sizeof *to; ++i)
        if (!(*to[i] = PyUnicode_InternFromString(text[i]))) return -1;
    return PyModule_AddFunctions(module, methods);
}

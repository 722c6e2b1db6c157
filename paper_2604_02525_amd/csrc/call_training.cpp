// The host side of the training operators' calls: arguments out of their Python objects, checked against each other, missing outputs
// allocated, the C entry point.  Through ctypes and torch's Python functions the call of the block norm took 11.9 us, its backward 30, while their kernels take
// 4 to 6 on a few rows; here the two calls take 5.4 and 7.6 us, their launches among them.
#include "call_common.h"

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

struct names_t {
    PyObject *a, *ckpt_g, *ckpt_u, *d_g, *d_u, *s, *h, *rstd_post, *rstd_pre, *ckpt_y, *ckpt_s, *d_x, *d_y, *d_w_post, *d_w_pre, *d_gate;
} name;

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

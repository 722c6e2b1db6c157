// extern "C" entry points of the training operators around the products (block norm, gated activation, 8-bit checkpoints and the weight
// gradient from one): argument validation, before any HIP call.
#include <math.h>

#include "common.h"

namespace adahop {

namespace {

constexpr int64_t MAX_EXTENT = (int64_t)1 << 21, MAX_NORM_COLS = 16384;

bool valid_shape(int64_t rows, int64_t cols)
{
    return rows >= 0 && rows <= MAX_EXTENT && cols >= 1 && cols <= MAX_EXTENT && rows * cols < ((int64_t)1 << 35);
}

bool present(const adahop_tensor_t &t) { return t.data != nullptr; }
bool present(const adahop_ckpt8_t &k) { return k.codes != nullptr || k.scales != nullptr; }

// A [rows, cols] tensor as described: absent, or aligned to its elements with rows that do not overlap.
bool valid(const adahop_tensor_t &t, int64_t cols)
{
    if (!present(t)) return true;
    return (t.f32 == 0 || t.f32 == 1) && t.ld >= cols && t.ld < ((int64_t)1 << 40) && aligned(t.data, t.f32 ? 4 : 2);
}

bool valid_vector(const adahop_tensor_t &t) { return !present(t) || ((t.f32 == 0 || t.f32 == 1) && aligned(t.data, t.f32 ? 4 : 2)); }

bool valid(const adahop_ckpt8_t &k, int64_t cols)
{
    if (!present(k)) return true;
    return k.codes && k.scales && aligned(k.codes, 16) && k.ld_codes >= cols && k.ld_codes % 16 == 0 && k.ld_scales >= ceil_div(cols, 32) &&
           k.ld_codes < ((int64_t)1 << 40) && k.ld_scales < ((int64_t)1 << 40);
}

bool same_type(const adahop_tensor_t &a, const adahop_tensor_t &b) { return !present(a) || !present(b) || a.f32 == b.f32; }

} // namespace

} // namespace adahop

using namespace adahop;

extern "C" {

int adahop_ckpt8_pack(int64_t rows, int64_t cols, const adahop_tensor_t *x, const adahop_ckpt8_t *out, void *stream)
{
    if (!x || !out || !valid_shape(rows, cols)) return ADAHOP_E_INVALID_ARG;
    if (rows == 0) return ADAHOP_OK;
    if (!present(*x) || !present(*out) || !valid(*x, cols) || !valid(*out, cols)) return ADAHOP_E_INVALID_ARG;
    return launch_ckpt8_pack(rows, cols, *x, *out, static_cast<hipStream_t>(stream));
}

int adahop_ckpt8_unpack(int64_t rows, int64_t cols, const adahop_ckpt8_t *x, const adahop_tensor_t *col_scale, const adahop_tensor_t *out, void *stream)
{
    if (!x || !out || !valid_shape(rows, cols)) return ADAHOP_E_INVALID_ARG;
    if (rows == 0) return ADAHOP_OK;
    const adahop_tensor_t scale = col_scale ? *col_scale : adahop_tensor_t{};
    if (!present(*x) || !present(*out) || !valid(*x, cols) || !valid(*out, cols) || !valid_vector(scale)) return ADAHOP_E_INVALID_ARG;
    return launch_ckpt8_unpack(rows, cols, *x, scale, *out, static_cast<hipStream_t>(stream));
}

int adahop_swiglu(const adahop_swiglu_t *p, void *stream)
{
    if (!p || !valid_shape(p->rows, p->cols)) return ADAHOP_E_INVALID_ARG;
    if (p->rows == 0) return ADAHOP_OK;
    if (!present(p->g) || !present(p->u) || p->g.f32 != p->u.f32 || !present(p->a)) return ADAHOP_E_INVALID_ARG;
    if (!valid(p->g, p->cols) || !valid(p->u, p->cols) || !valid(p->a, p->cols) || !valid(p->ckpt_g, p->cols) || !valid(p->ckpt_u, p->cols))
        return ADAHOP_E_INVALID_ARG;
    return launch_swiglu(*p, static_cast<hipStream_t>(stream));
}

int adahop_swiglu_backward(const adahop_swiglu_t *p, void *stream)
{
    if (!p || !valid_shape(p->rows, p->cols)) return ADAHOP_E_INVALID_ARG;
    if (p->rows == 0) return ADAHOP_OK;
    const bool kept = present(p->ckpt_g);
    if (kept != present(p->ckpt_u)) return ADAHOP_E_INVALID_ARG;
    if (!kept && (!present(p->g) || !present(p->u))) return ADAHOP_E_INVALID_ARG;
    if (!present(p->d_a) || !present(p->d_g) || !present(p->d_u)) return ADAHOP_E_INVALID_ARG;
    for (const adahop_tensor_t *t : {&p->g, &p->u, &p->a, &p->d_a, &p->d_g, &p->d_u})
        if (!valid(*t, p->cols)) return ADAHOP_E_INVALID_ARG;
    for (const adahop_ckpt8_t *k : {&p->ckpt_g, &p->ckpt_u, &p->ckpt_a})
        if (!valid(*k, p->cols)) return ADAHOP_E_INVALID_ARG;
    return launch_swiglu_backward(*p, static_cast<hipStream_t>(stream));
}

// What both directions of the block norm have in common.
static bool valid_block_norm(const adahop_block_norm_t *p)
{
    if (!p || !valid_shape(p->rows, p->cols) || p->cols > MAX_NORM_COLS) return false;
    if ((p->post_norm != 0 && p->post_norm != 1) || !isfinite(p->residual_scale) || !isfinite(p->branch_scale)) return false;
    if (!valid_vector(p->w_post) || !valid_vector(p->w_pre)) return false;
    if (present(p->gate)) {
        if (!valid(p->gate, p->cols) || p->gate_rows < 1 || p->gates < 0 || p->gate_rows > MAX_EXTENT || p->gates > MAX_EXTENT) return false;
        if (p->gates * p->gate_rows < p->rows) return false;
    }
    for (const float *f : {p->rstd_post, p->rstd_pre, p->d_w_post, p->d_w_pre})
        if (!aligned(f, 4)) return false;
    for (const adahop_tensor_t *t : {&p->x, &p->y, &p->s, &p->h, &p->d_s, &p->d_h, &p->d_x, &p->d_y, &p->d_gate})
        if (!valid(*t, p->cols)) return false;
    return valid(p->ckpt_y, p->cols) && valid(p->ckpt_s, p->cols);
}

int adahop_block_norm(const adahop_block_norm_t *p, void *stream)
{
    if (!valid_block_norm(p) || !(p->eps > 0.0f) || !isfinite(p->eps)) return ADAHOP_E_INVALID_ARG;
    if (p->rows == 0) return ADAHOP_OK;
    if (!present(p->x) && !present(p->y)) return ADAHOP_E_INVALID_ARG;
    if (!present(p->s) && !present(p->h)) return ADAHOP_E_INVALID_ARG;
    if (!same_type(p->x, p->s)) return ADAHOP_E_INVALID_ARG;
    if ((present(p->ckpt_y) || p->post_norm || present(p->gate)) && !present(p->y)) return ADAHOP_E_INVALID_ARG;
    if (p->rstd_post && !p->post_norm) return ADAHOP_E_INVALID_ARG;
    if ((present(p->ckpt_s) || p->rstd_pre) && !present(p->h)) return ADAHOP_E_INVALID_ARG;
    adahop_block_norm_t q = *p;
    if (!present(q.y)) q.w_post = {}; // whatever it holds: no branch, nothing of it in s
    return launch_block_norm(q, static_cast<hipStream_t>(stream));
}

size_t adahop_block_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t gate_rows)
{
    if (!valid_shape(rows, cols) || cols > MAX_NORM_COLS || gate_rows < 0) return 0;
    return block_norm_backward_workspace_bytes(rows, cols, gate_rows);
}

int adahop_block_norm_backward(const adahop_block_norm_t *p, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!valid_block_norm(p)) return ADAHOP_E_INVALID_ARG;
    if (present(p->d_gate) && !present(p->gate)) return ADAHOP_E_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (p->rows == 0) return launch_block_norm_no_rows(*p, st);
    if (!present(p->d_s) && !present(p->d_h)) return ADAHOP_E_INVALID_ARG;
    const bool kept_s = present(p->ckpt_s), kept_y = present(p->ckpt_y);
    const bool needs_y = p->post_norm || p->d_w_post || present(p->d_gate);
    if (present(p->d_h) && (!p->rstd_pre || (!kept_s && !present(p->s)))) return ADAHOP_E_INVALID_ARG;
    if (p->d_w_pre && !present(p->d_h)) return ADAHOP_E_INVALID_ARG;
    if (needs_y && !kept_y && !present(p->y)) return ADAHOP_E_INVALID_ARG;
    if (p->post_norm && !p->rstd_post) return ADAHOP_E_INVALID_ARG;
    // both saved tensors are 8-bit checkpoints, or neither is
    if (present(p->d_h) && needs_y && kept_s != kept_y) return ADAHOP_E_INVALID_ARG;
    const bool kept = present(p->d_h) ? kept_s : kept_y;
    // one type for the residual stream and its gradients, one for the block's side
    const adahop_tensor_t none = {}, *stream_side[] = {&p->d_s, &p->d_x, kept ? &none : &p->s}, *block_side[] = {&p->d_h, &p->d_y, kept ? &none : &p->y};
    int s32 = -1, y32 = -1;
    for (const adahop_tensor_t *t : stream_side)
        if (present(*t)) {
            if (s32 >= 0 && s32 != t->f32) return ADAHOP_E_INVALID_ARG;
            s32 = t->f32;
        }
    for (const adahop_tensor_t *t : block_side)
        if (present(*t)) {
            if (y32 >= 0 && y32 != t->f32) return ADAHOP_E_INVALID_ARG;
            y32 = t->f32;
        }
    const size_t need = block_norm_backward_workspace_bytes(p->rows, p->cols, present(p->gate) ? p->gate_rows : 0);
    if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return ADAHOP_E_WORKSPACE;
    adahop_block_norm_t q = *p;
    if (!present(q.d_h)) q.w_pre = {}; // as above
    return launch_block_norm_backward(q, s32 == 1, y32 == 1, kept, workspace, st);
}

size_t adahop_ckpt8_wgrad_workspace_bytes(int64_t tokens, int64_t d_out, int64_t d_in)
{
    if (!valid_shape(tokens, d_out) || !valid_shape(tokens, d_in) || !valid_shape(d_out, d_in) || d_out < 1) return 0;
    return wgrad8_workspace_bytes(tokens, d_out, d_in);
}

int adahop_debug_ckpt8_wgrad_plan(int64_t tokens, int64_t d_out, int64_t d_in, int *tile, int *shares, int *slices)
{
    if (!valid_shape(tokens, d_out) || !valid_shape(tokens, d_in) || !valid_shape(d_out, d_in) || d_out < 1 || !tile || !shares || !slices) return ADAHOP_E_INVALID_ARG;
    wgrad8_plan(tokens, d_out, d_in, tile, shares, slices);
    return ADAHOP_OK;
}

int adahop_ckpt8_wgrad(int64_t tokens, int64_t d_out, int64_t d_in, const adahop_tensor_t *G, const adahop_ckpt8_t *x, const adahop_tensor_t *col_scale,
                       const adahop_tensor_t *add, const adahop_tensor_t *C, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!G || !x || !C || !valid_shape(tokens, d_out) || !valid_shape(tokens, d_in) || !valid_shape(d_out, d_in) || d_out < 1) return ADAHOP_E_INVALID_ARG;
    const adahop_tensor_t none = {}, scale = col_scale ? *col_scale : none, sum = add ? *add : none;
    if (!present(*C) || !valid(*C, d_in) || !valid_vector(scale) || !valid(sum, d_in)) return ADAHOP_E_INVALID_ARG;
    if (tokens > 0) {
        if (!present(*G) || G->f32 != 0 || !valid(*G, d_out) || G->ld % 8 != 0 || !aligned(G->data, 16)) return ADAHOP_E_INVALID_ARG;
        if (!present(*x) || !valid(*x, d_in)) return ADAHOP_E_INVALID_ARG;
        // a stage's 32 rows of G are addressed by 32 bits; the checkpoint, expanded row by row, has the same limit
        if (G->ld >= ((int64_t)1 << 25) || x->ld_codes >= ((int64_t)1 << 25) || x->ld_scales >= ((int64_t)1 << 25)) return ADAHOP_E_INVALID_ARG;
    }
    const size_t need = wgrad8_workspace_bytes(tokens, d_out, d_in);
    if (need && (!workspace || !aligned(workspace, 256) || workspace_bytes < need)) return ADAHOP_E_WORKSPACE;
    return launch_wgrad8(tokens, d_out, d_in, *G, *x, scale, sum, *C, workspace, static_cast<hipStream_t>(stream));
}

} // extern "C"

// extern "C" entry points of what a training step does behind the last block (loss over a vocabulary, orthogonalised updates): argument validation, before any HIP call.
#include <math.h>

#include "common.h"

namespace adahop {

namespace {

constexpr int64_t MAX_EXTENT = (int64_t)1 << 21, MAX_ELEMENTS = (int64_t)1 << 35, MAX_LD = (int64_t)1 << 40;
constexpr int64_t MAX_SIDE = (int64_t)1 << 16, MAX_MATRIX = (int64_t)1 << 31, MAX_OPERAND_LD = (int64_t)1 << 22, MAX_MATRIX_LD = (int64_t)1 << 26;
constexpr int MAX_STEPS = 64;

bool present(const adahop_tensor_t &t) { return t.data != nullptr; }

bool valid(const adahop_tensor_t &t, int64_t cols, int64_t max_ld = MAX_LD)
{
    if (!present(t)) return true;
    return (t.f32 == 0 || t.f32 == 1) && t.ld >= cols && t.ld < max_ld && aligned(t.data, t.f32 ? 4 : 2);
}

bool valid_extents(int64_t tokens, int64_t vocab, int64_t dim)
{
    if (tokens < 0 || tokens > MAX_EXTENT || vocab < 1 || vocab > MAX_EXTENT || dim < 1 || dim > MAX_EXTENT) return false;
    return tokens * dim < MAX_ELEMENTS && vocab * dim < MAX_ELEMENTS && tokens * vocab < MAX_ELEMENTS;
}

bool valid_loss(const adahop_linear_ce_t *p)
{
    if (!p || !valid_extents(p->tokens, p->vocab, p->dim)) return false;
    for (const adahop_tensor_t *t : {&p->h, &p->w})
        if (t->f32 || t->ld < p->dim || t->ld >= MAX_OPERAND_LD || !aligned(t->data, 2)) return false;
    return isfinite(p->logit_scale) && isfinite(p->z_loss);
}

// What both directions read, where there are tokens.
bool has_operands(const adahop_linear_ce_t &p) { return present(p.h) && present(p.w) && p.targets && aligned(p.targets, 8); }

bool valid_sides(int64_t rows, int64_t cols) { return rows >= 1 && rows <= MAX_SIDE && cols >= 1 && cols <= MAX_SIDE && rows * cols < MAX_MATRIX; }

bool valid_method(const adahop_newton_schulz_t *m)
{
    if (!m || !valid_sides(m->rows, m->cols)) return false;
    for (const float f : {m->a, m->b, m->c, m->eps, m->scale})
        if (!isfinite(f)) return false;
    return m->steps >= 1 && m->steps <= MAX_STEPS && m->eps >= 0.0f;
}

bool holds(void *workspace, size_t bytes, size_t need) { return !need || (workspace && aligned(workspace, 256) && bytes >= need); }

} // namespace

} // namespace adahop

using namespace adahop;

extern "C" {

size_t adahop_linear_ce_workspace_bytes(const adahop_linear_ce_t *p, int backward)
{
    return valid_loss(p) && p->tokens > 0 ? linear_ce_workspace_bytes(*p, backward != 0) : 0;
}

int adahop_linear_ce(const adahop_linear_ce_t *p, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!valid_loss(p) || !aligned(p->loss, 4) || !aligned(p->lse, 4)) return ADAHOP_E_INVALID_ARG;
    if (p->tokens == 0) return ADAHOP_OK;
    if (!has_operands(*p) || (!p->loss && !p->lse)) return ADAHOP_E_INVALID_ARG;
    if (!holds(workspace, workspace_bytes, linear_ce_workspace_bytes(*p, false))) return ADAHOP_E_WORKSPACE;
    return launch_linear_ce(*p, workspace, static_cast<hipStream_t>(stream));
}

int adahop_linear_ce_backward(const adahop_linear_ce_t *p, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!valid_loss(p) || !valid(p->d_h, p->dim) || !valid(p->d_w, p->dim) || !valid(p->add, p->dim)) return ADAHOP_E_INVALID_ARG;
    if (p->tokens == 0) return present(p->d_w) ? launch_linear_ce_no_tokens(*p, static_cast<hipStream_t>(stream)) : ADAHOP_OK;
    if (!has_operands(*p) || !p->lse || !aligned(p->lse, 4) || !aligned(p->d_loss, 4) || (!present(p->d_h) && !present(p->d_w))) return ADAHOP_E_INVALID_ARG;
    if (p->d_loss && (p->d_loss_stride < 0 || p->d_loss_stride >= MAX_LD)) return ADAHOP_E_INVALID_ARG;
    if (present(p->add) && !present(p->d_w)) return ADAHOP_E_INVALID_ARG;
    if (!holds(workspace, workspace_bytes, linear_ce_workspace_bytes(*p, true))) return ADAHOP_E_WORKSPACE;
    return launch_linear_ce_backward(*p, workspace, static_cast<hipStream_t>(stream));
}

size_t adahop_newton_schulz_workspace_bytes(int64_t rows, int64_t cols)
{
    return valid_sides(rows, cols) ? newton_schulz_workspace_bytes(rows, cols) : 0;
}

int adahop_orthogonalize(const adahop_newton_schulz_t *method, const adahop_tensor_t *g, const adahop_tensor_t *out, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    if (!valid_method(method) || !g || !out || !present(*g) || !present(*out) || !valid(*g, method->cols, MAX_MATRIX_LD) || !valid(*out, method->cols, MAX_MATRIX_LD)) return ADAHOP_E_INVALID_ARG;
    if (!holds(workspace, workspace_bytes, newton_schulz_workspace_bytes(method->rows, method->cols))) return ADAHOP_E_WORKSPACE;
    return launch_newton_schulz(*method, *g, *out, nullptr, workspace, static_cast<hipStream_t>(stream));
}

int adahop_muon_update(const adahop_newton_schulz_t *method, const adahop_muon_t *p, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!valid_method(method) || !p || p->rows != method->rows || p->cols != method->cols) return ADAHOP_E_INVALID_ARG;
    for (const adahop_tensor_t *t : {&p->g, &p->momentum, &p->momentum_out, &p->w, &p->w_out})
        if (!present(*t) || !valid(*t, p->cols, MAX_MATRIX_LD)) return ADAHOP_E_INVALID_ARG;
    if (!valid(p->w_bf16, p->cols, MAX_MATRIX_LD) || (present(p->w_bf16) && p->w_bf16.f32)) return ADAHOP_E_INVALID_ARG;
    if (!p->momentum.f32 || !p->momentum_out.f32 || p->w.f32 != p->w_out.f32) return ADAHOP_E_INVALID_ARG;
    if (!isfinite(p->rate) || !isfinite(p->mu) || !isfinite(p->weight_decay) || (p->nesterov != 0 && p->nesterov != 1)) return ADAHOP_E_INVALID_ARG;
    if (!holds(workspace, workspace_bytes, newton_schulz_workspace_bytes(p->rows, p->cols))) return ADAHOP_E_WORKSPACE;
    return launch_newton_schulz(*method, p->g, {}, p, workspace, static_cast<hipStream_t>(stream));
}

int adahop_debug_linear_ce_plan(int64_t tokens, int64_t vocab, int64_t dim, int product, int *tile, int *alone, int *slices)
{
    if (!valid_extents(tokens, vocab, dim) || tokens < 1 || product < 0 || product > 2 || !tile || !alone || !slices) return ADAHOP_E_INVALID_ARG;
    linear_ce_plan(tokens, vocab, dim, product, tile, alone, slices);
    return ADAHOP_OK;
}

int adahop_debug_newton_schulz_plan(int64_t rows, int64_t cols, int product, int *tile, int *alone, int *slices)
{
    if (!valid_sides(rows, cols) || product < 0 || product > 2 || !tile || !alone || !slices) return ADAHOP_E_INVALID_ARG;
    newton_schulz_plan(rows, cols, product, tile, alone, slices);
    return ADAHOP_OK;
}

} // extern "C"

// Backward of the norms around a block (block_norm.hip).  With t = w_pre * dh, q = beta gate * w_post and D columns:
//
//     d  = ds + r_s (t - shat mean(t shat))               gradient of s
//     dx = alpha d,   dy = r_y (q d - yhat mean(q d yhat))
//     dw_pre = sum_rows dh shat,   dw_post = sum_rows beta gate d yhat,   dgate = sum over the gate row's rows of beta w_post d yhat
//
// d enters the second mean, which would make one sum over the row wait for the other.  Written out,
//     sum(q d yhat) = sum(q yhat (ds + r_s t)) - r_s mean(t shat) sum(q yhat shat),
// three sums that are formed together: one barrier for a row.
//
// A workgroup takes a run of rows one after the other and keeps its columns' part of the three weight gradients in registers; they go
// to the workspace once per run and k_block_norm_reduce adds the runs up, in their order: the same bits every time.  Bound by the memory.
#include "ckpt8.h"
#include "row_sums.h"

namespace adahop {

namespace {

// Runs of rows.  A gate row that stands for `group` rows: either a run is several whole groups (their gate gradients are complete
// when their last row is done), or a group is cut into `cuts` runs, whose parts are added up afterwards.
struct runs_t {
    int64_t group, rows, number; // rows per group; rows per run; runs
    int cuts;                    // runs per group, 0: whole groups
};

constexpr int64_t COMPUTE_UNITS = 256;

int threads_of(int64_t cols)
{
    const int64_t pieces = ceil_div(cols, 8);
    return (int)(pieces > ROW_THREADS ? ROW_THREADS : ceil_div(pieces, 64) * 64);
}

runs_t runs_of(int64_t rows, int64_t cols, int64_t gate_rows)
{
    runs_t r;
    r.group = gate_rows > 0 && gate_rows < rows ? gate_rows : rows;
    const int64_t want = ceil_div(rows, COMPUTE_UNITS * (ROW_THREADS / threads_of(cols)));
    if (r.group <= want) {
        r.rows = want / r.group * r.group;
        r.cuts = 0;
        r.number = ceil_div(rows, r.rows);
    } else {
        r.rows = ceil_div(r.group, ceil_div(r.group, want));
        r.cuts = (int)ceil_div(r.group, r.rows);
        r.number = ceil_div(rows, r.group) * r.cuts;
    }
    return r;
}

struct backward_t {
    adahop_block_norm_t q;
    runs_t runs;
    float *part; // [3][runs][cols]: w_pre, w_post, gate; nullptr: one run, whose sums are the results
};

template <bool KEPT, bool F32> struct saved8 { // eight saved values of a row: from an 8-bit checkpoint, or from a tensor
    raw8<F32> r;
};
template <bool F32> struct saved8<true, F32> {
    packed8 r;
};

template <bool KEPT, bool F32> __device__ __forceinline__ void load_saved(saved8<KEPT, F32> &o, const adahop_ckpt8_t &k, const adahop_tensor_t &t, int64_t row, int c, int n)
{
    if constexpr (KEPT)
        o.r = load_packed8(k, row, c, n);
    else
        o.r = load8<F32>(t.data, row * t.ld + c, n);
}

template <bool KEPT, bool F32> __device__ __forceinline__ void widen_saved(const saved8<KEPT, F32> &o, float r, float (&v)[8])
{
    if constexpr (KEPT) {
        unpack8(o.r, v);
    } else {
        widen8(o.r, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= r;
    }
}

// C: pieces of 8 columns per lane; SF32: ds, dx and a saved s are fp32; YF32: dh, dy and a saved y are.
template <int C, bool KEPT, bool SF32, bool YF32> __global__ __launch_bounds__(ROW_THREADS) void k_block_norm_backward(backward_t b)
{
    __shared__ row_sums_t<3> lds;
    const adahop_block_norm_t &q = b.q;
    const int threads = blockDim.x, waves = threads >> 6;
    int turn = 0;
    const auto col = [&](int j) { return (int)(threadIdx.x + j * threads) * 8; };
    const auto left = [&](int j) { return (int)q.cols - col(j); };
    float wpost[C][8], wpre[C][8], gate[C][8], apre[C][8], apost[C][8], agate[C][8];
#pragma unroll
    for (int j = 0; j < C; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            wpost[j][i] = wpre[j][i] = gate[j][i] = 1.0f;
            apre[j][i] = apost[j][i] = agate[j][i] = 0.0f;
        }
        if (left(j) > 0) {
            if (q.w_post.data) load8_any(q.w_post, col(j), left(j), wpost[j]);
            if (q.w_pre.data) load8_any(q.w_pre, col(j), left(j), wpre[j]);
        }
    }
    int64_t row = blockIdx.x * b.runs.rows, end = row + b.runs.rows;
    if (b.runs.cuts) {
        const int64_t g = blockIdx.x / b.runs.cuts, cut = blockIdx.x % b.runs.cuts;
        row = g * b.runs.group + cut * b.runs.rows;
        end = row + b.runs.rows < (g + 1) * b.runs.group ? row + b.runs.rows : (g + 1) * b.runs.group;
    }
    if (end > q.rows) end = q.rows;
    const float over_cols = 1.0f / (float)q.cols;
    const bool has_h = q.d_h.data, has_y = KEPT ? q.ckpt_y.codes != nullptr : q.y.data != nullptr;
    int64_t gate_row = -1;
    for (; row < end; ++row) {
        if (q.gate.data && row / q.gate_rows != gate_row) {
            gate_row = row / q.gate_rows;
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (left(j) > 0) load8_any(q.gate, gate_row * q.gate.ld + col(j), left(j), gate[j]);
        }
        float ds[C][8], t[C][8], shat[C][8], yhat[C][8], sum[3] = {0.0f, 0.0f, 0.0f};
        const float rs = has_h ? q.rstd_pre[row] : 0.0f, ry = q.post_norm ? q.rstd_post[row] : 1.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            raw8<SF32> rds = zero8<SF32>();
            raw8<YF32> rdh = zero8<YF32>();
#pragma unroll
            for (int i = 0; i < 8; ++i) shat[j][i] = yhat[j][i] = 0.0f;
            if (left(j) > 0) {
                if (q.d_s.data) rds = load8<SF32>(q.d_s.data, row * q.d_s.ld + col(j), left(j));
                if (has_h) {
                    rdh = load8<YF32>(q.d_h.data, row * q.d_h.ld + col(j), left(j));
                    saved8<KEPT, SF32> k;
                    load_saved(k, q.ckpt_s, q.s, row, col(j), left(j));
                    widen_saved(k, rs, shat[j]);
                }
                if (has_y) {
                    saved8<KEPT, YF32> k;
                    load_saved(k, q.ckpt_y, q.y, row, col(j), left(j));
                    widen_saved(k, ry, yhat[j]);
                }
            }
            widen8(rds, ds[j]);
            widen8(rdh, t[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                apre[j][i] = __builtin_fmaf(t[j][i], shat[j][i], apre[j][i]);
                t[j][i] *= wpre[j][i];
                const float m = q.branch_scale * gate[j][i] * wpost[j][i] * yhat[j][i];
                sum[0] = __builtin_fmaf(t[j][i], shat[j][i], sum[0]);
                sum[1] = __builtin_fmaf(m, __builtin_fmaf(rs, t[j][i], ds[j][i]), sum[1]);
                sum[2] = __builtin_fmaf(m, shat[j][i], sum[2]);
            }
        }
        row_sums(lds, turn, waves, sum);
        const float c1 = sum[0] * over_cols, c2 = q.post_norm ? (sum[1] - rs * c1 * sum[2]) * over_cols : 0.0f;
        const bool gate_ends = !b.runs.cuts && (row + 1 == end || (row + 1) % b.runs.group == 0);
#pragma unroll
        for (int j = 0; j < C; ++j) {
            float dx[8], dy[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = __builtin_fmaf(rs, __builtin_fmaf(-c1, shat[j][i], t[j][i]), ds[j][i]), u = q.branch_scale * d, uy = u * yhat[j][i];
                dx[i] = q.residual_scale * d;
                dy[i] = ry * __builtin_fmaf(-c2, yhat[j][i], u * gate[j][i] * wpost[j][i]);
                apost[j][i] = __builtin_fmaf(uy, gate[j][i], apost[j][i]);
                agate[j][i] = __builtin_fmaf(uy, wpost[j][i], agate[j][i]);
            }
            if (left(j) > 0) {
                if (q.d_x.data) store8<SF32>(q.d_x.data, row * q.d_x.ld + col(j), left(j), dx);
                if (q.d_y.data) store8<YF32>(q.d_y.data, row * q.d_y.ld + col(j), left(j), dy);
                if (gate_ends && q.d_gate.data) store8_any(q.d_gate, row / q.gate_rows * q.d_gate.ld + col(j), left(j), agate[j]);
            }
            if (gate_ends) {
#pragma unroll
                for (int i = 0; i < 8; ++i) agate[j][i] = 0.0f;
            }
        }
    }
    const int64_t one = b.runs.number * q.cols, at = blockIdx.x * q.cols;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        if (left(j) <= 0) continue;
        if (q.d_w_pre) store8<true>(b.part ? b.part + at : q.d_w_pre, col(j), left(j), apre[j]);
        if (q.d_w_post) store8<true>(b.part ? b.part + one + at : q.d_w_post, col(j), left(j), apost[j]);
        if (q.d_gate.data && b.runs.cuts) {
            if (b.part)
                store8<true>(b.part + 2 * one + at, col(j), left(j), agate[j]);
            else
                store8_any(q.d_gate, col(j), left(j), agate[j]);
        }
    }
}

// Sums of the runs' parts.  blockIdx.y = 0, 1: the weight gradients; from 2 on the gate rows.  A workgroup takes 64 columns; its waves share
// the runs, each in order, and their sums are added in order.
constexpr int REDUCE_WAVES = 8;

__global__ __launch_bounds__(64 * REDUCE_WAVES) void k_block_norm_reduce(backward_t b)
{
    __shared__ float lds[REDUCE_WAVES][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, which = blockIdx.y < 2 ? blockIdx.y : 2;
    float *const to = which == 0 ? b.q.d_w_pre : which == 1 ? b.q.d_w_post : nullptr;
    if (which < 2 ? !to : !b.q.d_gate.data) return; // of the whole workgroup
    const int64_t c = (int64_t)blockIdx.x * 64 + lane, first = which < 2 ? 0 : (int64_t)(blockIdx.y - 2) * b.runs.cuts;
    const int64_t runs = which < 2 ? b.runs.number : b.runs.cuts, share = (runs + REDUCE_WAVES - 1) / REDUCE_WAVES;
    const int64_t begin = w * share, end = begin + share < runs ? begin + share : runs;
    float sum = 0.0f;
    if (c < b.q.cols) {
        const float *p = b.part + (which * b.runs.number + first + begin) * b.q.cols + c;
#pragma unroll 8
        for (int64_t i = begin; i < end; ++i, p += b.q.cols) sum += *p;
    }
    lds[w][lane] = sum;
    __syncthreads();
    if (w || c >= b.q.cols) return;
#pragma unroll
    for (int i = 1; i < REDUCE_WAVES; ++i) sum += lds[i][lane];
    if (which < 2)
        to[c] = sum;
    else if (b.q.d_gate.f32)
        static_cast<float *>(b.q.d_gate.data)[(int64_t)(blockIdx.y - 2) * b.q.d_gate.ld + c] = sum;
    else
        static_cast<uint16_t *>(b.q.d_gate.data)[(int64_t)(blockIdx.y - 2) * b.q.d_gate.ld + c] = (uint16_t)bf16_pair(sum, 0.0f);
}

// d_gate's rows from `from` on, and (from == 0) the weight gradients: no row of the operand has a part in them.
__global__ __launch_bounds__(256) void k_block_norm_zero(adahop_block_norm_t q, int64_t from)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= q.cols) return;
    if (from == 0 && blockIdx.y == 0) {
        if (q.d_w_pre) q.d_w_pre[c] = 0.0f;
        if (q.d_w_post) q.d_w_post[c] = 0.0f;
    }
    if (!q.d_gate.data) return;
    for (int64_t g = from + blockIdx.y; g < q.gates; g += gridDim.y) {
        if (q.d_gate.f32)
            static_cast<float *>(q.d_gate.data)[g * q.d_gate.ld + c] = 0.0f;
        else
            static_cast<uint16_t *>(q.d_gate.data)[g * q.d_gate.ld + c] = 0;
    }
}

int zero_from(const adahop_block_norm_t &q, int64_t from, hipStream_t st)
{
    const int64_t gates = q.d_gate.data ? q.gates - from : 0;
    k_block_norm_zero<<<dim3((unsigned)ceil_div(q.cols, 256), (unsigned)(gates < 1 ? 1 : gates > 1024 ? 1024 : gates)), 256, 0, st>>>(q, from);
    return check_launch();
}

template <int C, bool KEPT> void launch(const backward_t &b, bool s32, bool y32, int threads, hipStream_t st)
{
    const unsigned n = (unsigned)b.runs.number;
    if (s32)
        y32 ? k_block_norm_backward<C, KEPT, true, true><<<n, threads, 0, st>>>(b) : k_block_norm_backward<C, KEPT, true, false><<<n, threads, 0, st>>>(b);
    else
        y32 ? k_block_norm_backward<C, KEPT, false, true><<<n, threads, 0, st>>>(b) : k_block_norm_backward<C, KEPT, false, false><<<n, threads, 0, st>>>(b);
}

} // namespace

size_t block_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t gate_rows)
{
    if (rows == 0) return 0;
    const runs_t r = runs_of(rows, cols, gate_rows);
    return r.number == 1 ? 0 : (size_t)3 * r.number * cols * sizeof(float);
}

int launch_block_norm_no_rows(const adahop_block_norm_t &q, hipStream_t st) { return zero_from(q, 0, st); }

int launch_block_norm_backward(const adahop_block_norm_t &q, bool s32, bool y32, bool kept, void *workspace, hipStream_t st)
{
    backward_t b = {q, runs_of(q.rows, q.cols, q.gate.data ? q.gate_rows : 0), nullptr};
    if (b.runs.number > 1) b.part = static_cast<float *>(workspace);
    const int threads = threads_of(q.cols);
    if (q.cols > 8 * ROW_THREADS)
        kept ? launch<2, true>(b, s32, y32, threads, st) : launch<2, false>(b, s32, y32, threads, st);
    else
        kept ? launch<1, true>(b, s32, y32, threads, st) : launch<1, false>(b, s32, y32, threads, st);
    int rc = check_launch();
    if (rc == ADAHOP_OK && q.d_gate.data && q.gates > ceil_div(q.rows, q.gate_rows)) rc = zero_from(q, ceil_div(q.rows, q.gate_rows), st);
    if (rc != ADAHOP_OK || !b.part) return rc;
    const int64_t gates = q.d_gate.data && b.runs.cuts ? ceil_div(q.rows, b.runs.group) : 0;
    if (!q.d_w_pre && !q.d_w_post && !gates) return ADAHOP_OK;
    k_block_norm_reduce<<<dim3((unsigned)ceil_div(q.cols, 64), (unsigned)(2 + gates)), 64 * REDUCE_WAVES, 0, st>>>(b);
    return check_launch();
}

} // namespace adahop

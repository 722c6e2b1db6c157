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

template <bool KEPT, bool F32> __device__ __forceinline__ void none(saved8<KEPT, F32> &o)
{
    if constexpr (KEPT) {
        o.r.codes = 0;
        o.r.scale = 0;
    } else {
        o.r = zero8<F32>();
    }
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
//
// One accumulator serves both the gate and w_post: with A = sum(beta d yhat) over rows of one gate row, its gate gradient is w_post A and its part of
// w_post's is gate A.  CUT: all rows of the run are of one gate row.  The row's values stay as they were loaded over the barrier and are widened again behind it
// (half the registers).  Up to 8192 columns (C = 1) the weights stay in registers, and the next row is loaded meanwhile unless the saved tensors are
// fp32; above that the sums do not all fit the registers.
template <int C, bool KEPT, bool CUT, bool SF32, bool YF32> __global__ __launch_bounds__(ROW_THREADS) void k_block_norm_backward(backward_t b)
{
    // registers that a row takes as it lies in memory: two rows at a time where that leaves enough for the rest
    constexpr int RAW = (SF32 ? 8 : 4) + (YF32 ? 8 : 4) + (KEPT ? 6 : (SF32 ? 8 : 4) + (YF32 ? 8 : 4));
    constexpr bool AHEAD = C == 1 && RAW <= 22;
    __shared__ row_sums_t<3> lds;
    const adahop_block_norm_t &q = b.q;
    const int threads = blockDim.x, waves = threads >> 6;
    int turn = 0;
    const auto col = [&](int j) { return (int)(threadIdx.x + j * threads) * 8; };
    const auto left = [&](int j) { return (int)q.cols - col(j); };
    const auto vector_of = [&](const adahop_tensor_t &t, int64_t at, int j, float (&v)[8]) { // ones where there is none
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.0f;
        if (t.data && left(j) > 0) load8_any(t, at + col(j), left(j), v);
    };
    const auto branch_of = [&](int64_t gate_row, int j, float (&v)[8]) { // beta gate w_post
        float g[8];
        vector_of(q.gate, gate_row * q.gate.ld, j, g);
        vector_of(q.w_post, 0, j, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= q.branch_scale * g[i];
    };
    float wbranch[C][8], wpre[C][8], apre[C][8], apost[CUT ? 1 : C][8], agate[C][8]; // agate: A of the gate row at hand
#pragma unroll
    for (int j = 0; j < C; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            apre[j][i] = agate[j][i] = 0.0f;
            if constexpr (!CUT) apost[j][i] = 0.0f;
        }
        if constexpr (C == 1) vector_of(q.w_pre, 0, j, wpre[j]);
    }
    int64_t row = blockIdx.x * b.runs.rows, end = row + b.runs.rows;
    if constexpr (CUT) {
        const int64_t g = blockIdx.x / b.runs.cuts, cut = blockIdx.x % b.runs.cuts;
        row = g * b.runs.group + cut * b.runs.rows;
        end = row + b.runs.rows < (g + 1) * b.runs.group ? row + b.runs.rows : (g + 1) * b.runs.group;
    }
    if (end > q.rows) end = q.rows;
    const float over_cols = 1.0f / (float)q.cols;
    const bool has_h = q.d_h.data, has_y = KEPT ? q.ckpt_y.codes != nullptr : q.y.data != nullptr;
    raw8<SF32> ds[C];
    raw8<YF32> dh[C];
    saved8<KEPT, SF32> sk[C];
    saved8<KEPT, YF32> yk[C];
    float rs = 0.0f, ry = 1.0f;
    const auto load_row = [&](int64_t r) {
        if (has_h) rs = q.rstd_pre[r];
        if (q.post_norm) ry = q.rstd_post[r];
#pragma unroll
        for (int j = 0; j < C; ++j) {
            ds[j] = q.d_s.data && left(j) > 0 ? load8<SF32>(q.d_s.data, r * q.d_s.ld + col(j), left(j)) : zero8<SF32>();
            dh[j] = has_h && left(j) > 0 ? load8<YF32>(q.d_h.data, r * q.d_h.ld + col(j), left(j)) : zero8<YF32>();
            none(sk[j]);
            none(yk[j]);
            if (has_h && left(j) > 0) load_saved(sk[j], q.ckpt_s, q.s, r, col(j), left(j));
            if (has_y && left(j) > 0) load_saved(yk[j], q.ckpt_y, q.y, r, col(j), left(j));
        }
    };
    int64_t gate_row = 0, gate_until = row; // first row of another gate row than the present one
    if (row < end) load_row(row);
    while (row < end) {
        if (row >= gate_until) {
            gate_row = q.gate.data ? row / q.gate_rows : 0;
            gate_until = q.gate.data ? (gate_row + 1) * q.gate_rows : end;
            if constexpr (C == 1) {
#pragma unroll
                for (int j = 0; j < C; ++j) branch_of(gate_row, j, wbranch[j]);
            }
        }
        float sum[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < C; ++j) {
            float d[8], t[8], shat[8], yhat[8];
            if constexpr (C > 1) {
                vector_of(q.w_pre, 0, j, wpre[j]);
                branch_of(gate_row, j, wbranch[j]);
            }
            widen8(ds[j], d);
            widen8(dh[j], t);
            widen_saved(sk[j], rs, shat);
            widen_saved(yk[j], ry, yhat);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                t[i] *= wpre[j][i];
                const float m = wbranch[j][i] * yhat[i];
                sum[0] = __builtin_fmaf(t[i], shat[i], sum[0]);
                sum[1] = __builtin_fmaf(m, __builtin_fmaf(rs, t[i], d[i]), sum[1]);
                sum[2] = __builtin_fmaf(m, shat[i], sum[2]);
            }
        }
        raw8<SF32> ds0[C];
        raw8<YF32> dh0[C];
        saved8<KEPT, SF32> sk0[C];
        saved8<KEPT, YF32> yk0[C];
        const float rs0 = rs, ry0 = ry;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            ds0[j] = ds[j], dh0[j] = dh[j], sk0[j] = sk[j], yk0[j] = yk[j];
            keep_raw(ds0[j]), keep_raw(dh0[j]), keep_raw(sk0[j].r), keep_raw(yk0[j].r);
        }
        if constexpr (AHEAD) {
            if (row + 1 < end) load_row(row + 1);
        }
        row_sums(lds, turn, waves, sum);
        const float c1 = sum[0] * over_cols, c2 = q.post_norm ? (sum[1] - rs0 * c1 * sum[2]) * over_cols : 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            float d[8], t[8], shat[8], yhat[8], dx[8], dy[8];
            if constexpr (C > 1) {
                vector_of(q.w_pre, 0, j, wpre[j]);
                branch_of(gate_row, j, wbranch[j]);
            }
            widen8(ds0[j], d);
            widen8(dh0[j], t);
            widen_saved(sk0[j], rs0, shat);
            widen_saved(yk0[j], ry0, yhat);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                apre[j][i] = __builtin_fmaf(t[i], shat[i], apre[j][i]);
                d[i] = __builtin_fmaf(rs0, __builtin_fmaf(-c1, shat[i], t[i] * wpre[j][i]), d[i]);
                dx[i] = q.residual_scale * d[i];
                dy[i] = ry0 * __builtin_fmaf(-c2, yhat[i], d[i] * wbranch[j][i]);
                agate[j][i] = __builtin_fmaf(q.branch_scale * d[i], yhat[i], agate[j][i]);
            }
            if (left(j) > 0) {
                if (q.d_x.data) store8<SF32>(q.d_x.data, row * q.d_x.ld + col(j), left(j), dx);
                if (q.d_y.data) store8<YF32>(q.d_y.data, row * q.d_y.ld + col(j), left(j), dy);
            }
        }
        ++row;
        if constexpr (!CUT) {
            if (row == end || row == gate_until) { // the gate row is complete
#pragma unroll
                for (int j = 0; j < C; ++j) {
                    float g[8], w[8];
                    vector_of(q.gate, gate_row * q.gate.ld, j, g);
                    vector_of(q.w_post, 0, j, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        apost[j][i] = __builtin_fmaf(agate[j][i], g[i], apost[j][i]);
                        w[i] *= agate[j][i];
                        agate[j][i] = 0.0f;
                    }
                    if (q.d_gate.data && left(j) > 0) store8_any(q.d_gate, gate_row * q.d_gate.ld + col(j), left(j), w);
                }
            }
        }
        if constexpr (!AHEAD) {
            if (row < end) load_row(row);
        }
    }
    const int64_t one = b.runs.number * q.cols, at = blockIdx.x * q.cols;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        if (left(j) <= 0) continue;
        if (q.d_w_pre) store8<true>(b.part ? b.part + at : q.d_w_pre, col(j), left(j), apre[j]);
        float v[8];
        if constexpr (CUT) {
            vector_of(q.w_post, 0, j, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= agate[j][i];
            if (q.d_gate.data) {
                if (b.part)
                    store8<true>(b.part + 2 * one + at, col(j), left(j), v);
                else
                    store8_any(q.d_gate, col(j), left(j), v);
            }
            vector_of(q.gate, gate_row * q.gate.ld, j, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= agate[j][i];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = apost[j][i];
        }
        if (q.d_w_post) store8<true>(b.part ? b.part + one + at : q.d_w_post, col(j), left(j), v);
    }
}

// Sums of the runs' parts.  blockIdx.y = 0, 1: the weight gradients; from 2 on the gate rows.  A workgroup takes `strip` columns, 64 or 32;
// its threads of one column share the runs, each in order, and their sums are added in one order.  Bound by the way to memory and
// back: a thread's loads are on their way BATCH at a time.  Strips of 32 where the runs are many, us for the whole backward pass: 4000 runs of 512 columns
// 27.8 (64: 34.4), 2048 of 1024 32.8 (36.2); 802 of 2048 25.0 (23.1).
constexpr int REDUCE_THREADS = 1024, BATCH = 16;

__global__ __launch_bounds__(REDUCE_THREADS) void k_block_norm_reduce(backward_t b, int strip)
{
    typedef unsigned int v2u __attribute__((ext_vector_type(2)));
    __shared__ float lds[REDUCE_THREADS / 64][64];
    const int which = blockIdx.y < 2 ? blockIdx.y : 2;
    float *const to = which == 0 ? b.q.d_w_pre : which == 1 ? b.q.d_w_post : nullptr;
    if (which < 2 ? !to : !b.q.d_gate.data) return; // of the whole workgroup
    const int at = threadIdx.x & (strip - 1), slot = threadIdx.x / strip, slots = REDUCE_THREADS / strip;
    const int64_t c = (int64_t)blockIdx.x * strip + at, first = which < 2 ? 0 : (int64_t)(blockIdx.y - 2) * b.runs.cuts;
    const int64_t runs = which < 2 ? b.runs.number : b.runs.cuts, share = (runs + slots - 1) / slots;
    const int64_t begin = slot * share, end = begin + share < runs ? begin + share : runs;
    float sum = 0.0f;
    if (c < b.q.cols) {
        const float *p = b.part + (which * b.runs.number + first + begin) * b.q.cols + c;
        for (int64_t i = begin; i < end; i += BATCH, p += BATCH * b.q.cols) {
            float v[BATCH]; // where fewer are left, the first again
#pragma unroll
            for (int j = 0; j < BATCH; ++j) v[j] = p[(i + j < end ? j : 0) * b.q.cols];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) sum += i + j < end ? v[j] : 0.0f;
        }
    }
    if (strip == 32) { // the halves of a wave
        const v2u r = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
        sum = __uint_as_float(r.x) + __uint_as_float(r.y);
    }
    lds[threadIdx.x >> 6][threadIdx.x & 63] = sum;
    __syncthreads();
    if ((int)threadIdx.x >= strip || c >= b.q.cols) return;
#pragma unroll
    for (int i = 1; i < REDUCE_THREADS / 64; ++i) sum += lds[i][threadIdx.x];
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

template <int C, bool KEPT, bool CUT> void launch(const backward_t &b, bool s32, bool y32, int threads, hipStream_t st)
{
    const unsigned n = (unsigned)b.runs.number;
    if (s32)
        y32 ? k_block_norm_backward<C, KEPT, CUT, true, true><<<n, threads, 0, st>>>(b) : k_block_norm_backward<C, KEPT, CUT, true, false><<<n, threads, 0, st>>>(b);
    else
        y32 ? k_block_norm_backward<C, KEPT, CUT, false, true><<<n, threads, 0, st>>>(b) : k_block_norm_backward<C, KEPT, CUT, false, false><<<n, threads, 0, st>>>(b);
}

template <int C> void launch(const backward_t &b, bool s32, bool y32, bool kept, int threads, hipStream_t st)
{
    if (kept)
        b.runs.cuts ? launch<C, true, true>(b, s32, y32, threads, st) : launch<C, true, false>(b, s32, y32, threads, st);
    else
        b.runs.cuts ? launch<C, false, true>(b, s32, y32, threads, st) : launch<C, false, false>(b, s32, y32, threads, st);
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
        launch<2>(b, s32, y32, kept, threads, st);
    else
        launch<1>(b, s32, y32, kept, threads, st);
    int rc = check_launch();
    if (rc == ADAHOP_OK && q.d_gate.data && q.gates > ceil_div(q.rows, q.gate_rows)) rc = zero_from(q, ceil_div(q.rows, q.gate_rows), st);
    if (rc != ADAHOP_OK || !b.part) return rc;
    const int64_t gates = q.d_gate.data && b.runs.cuts ? ceil_div(q.rows, b.runs.group) : 0;
    if (!q.d_w_pre && !q.d_w_post && !gates) return ADAHOP_OK;
    const int strip = b.runs.number > 1024 ? 32 : 64;
    k_block_norm_reduce<<<dim3((unsigned)ceil_div(q.cols, strip), (unsigned)(2 + gates)), REDUCE_THREADS, 0, st>>>(b, strip);
    return check_launch();
}

} // namespace adahop

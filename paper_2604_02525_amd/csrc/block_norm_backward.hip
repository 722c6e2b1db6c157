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
// A workgroup takes a run of rows one after the other, or several runs beside each other where rows are short, and keeps its columns' part of the three
// weight gradients in registers.  At the end its runs are added up by way of LDS and go to the workspace, and k_block_norm_reduce adds the
// workgroups' parts up, all in one order: the same bits every time.  Bound by the memory: 16384 x 8192 from 8-bit checkpoints takes 256 to 272 us in
// all, 5.0 to 5.3 TB/s; 16384 x 4096 148 us (two workgroups per compute unit, 17 MB of parts to the workspace and back); 777 x 4091 with a gate for
// every row, the residual stream in fp32, 27.2 us: two rows one after the other, each waiting for its loads.
#include "ckpt8.h"
#include "row_sums.h"

namespace adahop {

namespace {

// Runs of rows.  A gate row that stands for `group` rows: either a run is several whole groups (their gate gradients are complete
// when their last row is done), or a group is cut into `cuts` runs, whose parts are added up afterwards.  Runs go beside each other in a workgroup where
// three or more fit: 8192 rows of 1024 in 27.5 us instead of 32.8, 12000 of 512 in 20.1 instead of 27.6.  Where two fit, two workgroups for a
// compute unit wait less for each other: 8192 x 4096 in 112 us, as one in 115.
struct runs_t {
    int64_t group, rows, number; // rows per group; rows per run; runs
    int cuts;                    // runs per group, 0: whole groups
    int beside;                  // runs per workgroup
    bool joined;                 // the runs of a workgroup belong to one group, if groups are cut
    int64_t workgroups() const { return ceil_div(number, beside); }
    int64_t gate_parts() const { return joined ? workgroups() : number; }
    int gate_cuts() const { return joined ? cuts / beside : cuts; } // parts per group
};

constexpr int64_t COMPUTE_UNITS = 256;

int64_t strips_of(int64_t cols) { return ceil_div(cols, 8 * ROW_THREADS); } // that a row is cut into

int threads_of(int64_t cols) { return (int)(ceil_div(ceil_div(cols, 8 * strips_of(cols)), 64) * 64); } // eight columns each

runs_t runs_of(int64_t rows, int64_t cols, int64_t gate_rows)
{
    runs_t r;
    r.group = gate_rows > 0 && gate_rows < rows ? gate_rows : rows;
    const int64_t fit = ROW_THREADS / threads_of(cols), each = ceil_div(rows, COMPUTE_UNITS);
    r.beside = (int)(fit <= 2 ? 1 : each < fit ? each : fit);
    const int64_t want = ceil_div(rows, COMPUTE_UNITS * fit);
    if (r.group <= want) {
        r.rows = want / r.group * r.group;
        r.cuts = 0;
        r.number = ceil_div(rows, r.rows);
    } else {
        r.cuts = (int)ceil_div(r.group, want);
        if (r.cuts > r.beside) r.cuts = (int)ceil_div(r.cuts, r.beside) * r.beside;
        r.rows = ceil_div(r.group, r.cuts);
        r.number = ceil_div(rows, r.group) * r.cuts;
    }
    r.joined = r.cuts % r.beside == 0;
    return r;
}

struct backward_t {
    adahop_block_norm_t q;
    runs_t runs;
    int threads, gate_cuts; // threads per row; runs.gate_cuts()
    int64_t workgroups;
    const float2 *means; // of every row, for rows in strips
    float *part;         // [workgroups][cols] w_pre, the same w_post, [runs.gate_parts()][cols] gate; nullptr: a single row, whose sums are the results
};

__device__ __forceinline__ void put(const adahop_tensor_t &t, int64_t at, float v)
{
    if (t.f32)
        static_cast<float *>(t.data)[at] = v;
    else
        static_cast<uint16_t *>(t.data)[at] = (uint16_t)bf16_pair(v, 0.0f);
}

template <bool KEPT, bool F32> struct saved8 { // eight saved values of a row: from an 8-bit checkpoint, or from a tensor
    raw8<F32> r;
};
template <bool F32> struct saved8<true, F32> {
    packed8 r;
};

template <bool ODD, bool KEPT, bool F32> __device__ __forceinline__ void load_saved(saved8<KEPT, F32> &o, const adahop_ckpt8_t &k, const adahop_tensor_t &t, int64_t row, int c, int n)
{
    if constexpr (KEPT)
        o.r = load_packed8<ODD>(k, row, c, n);
    else
        o.r = load8<F32, ODD>(t.data, row * t.ld + c, n);
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

// v = t's eight elements from `at` on, n of which exist; ones where there is no t.
template <bool ODD> __device__ __forceinline__ void vector_of(const adahop_tensor_t &t, int64_t at, int n, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 1.0f;
    if (t.data && n > 0) load8_any<ODD>(t, at, n, v);
}

// v = beta gate w_post at column c
template <bool ODD> __device__ __forceinline__ void branch_of(const adahop_block_norm_t &q, int64_t gate_row, int c, int n, float (&v)[8])
{
    float g[8];
    vector_of<ODD>(q.gate, gate_row * q.gate.ld + c, to_load(n, gate_row + 1 < q.gates, q.cols), g);
    vector_of<ODD>(q.w_post, c, n, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= q.branch_scale * g[i];
    if (ODD && n < 8) zero_from(n, v);
}

// What a lane reads of a row.
template <bool ODD, bool KEPT, bool SF32, bool YF32> struct piece_t {
    raw8<SF32> ds;
    raw8<YF32> dh;
    saved8<KEPT, SF32> s;
    saved8<KEPT, YF32> y;

    __device__ __forceinline__ void load(const adahop_block_norm_t &q, int64_t row, int c, int n)
    {
        n = to_load(n, row + 1 < q.rows, q.cols);
        ds = q.d_s.data && n > 0 ? load8<SF32, ODD>(q.d_s.data, row * q.d_s.ld + c, n) : zero8<SF32>();
        dh = q.d_h.data && n > 0 ? load8<YF32, ODD>(q.d_h.data, row * q.d_h.ld + c, n) : zero8<YF32>();
        none(s);
        none(y);
        if (q.d_h.data && n > 0) load_saved<ODD>(s, q.ckpt_s, q.s, row, c, n);
        if ((KEPT ? q.ckpt_y.codes != nullptr : q.y.data != nullptr) && n > 0) load_saved<ODD>(y, q.ckpt_y, q.y, row, c, n);
    }
    // The share in the three sums of the n elements that exist.
    __device__ __forceinline__ void add(int n, float rs, float ry, const float (&wpre)[8], const float (&wbranch)[8], float (&sum)[3]) const
    {
        float d[8], t[8], shat[8], yhat[8];
        widen8(ds, d);
        widen8(dh, t);
        widen_saved(s, rs, shat);
        widen_saved(y, ry, yhat);
        if (ODD && n < 8) zero_from(n, d), zero_from(n, t), zero_from(n, shat), zero_from(n, yhat);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            t[i] *= wpre[i];
            const float m = wbranch[i] * yhat[i];
            sum[0] = __builtin_fmaf(t[i], shat[i], sum[0]);
            sum[1] = __builtin_fmaf(m, __builtin_fmaf(rs, t[i], d[i]), sum[1]);
            sum[2] = __builtin_fmaf(m, shat[i], sum[2]);
        }
    }
};

// mean(t shat) and mean(q yhat d) of a row
__device__ __forceinline__ float2 means_of(const adahop_block_norm_t &q, float rs, const float (&sum)[3])
{
    const float over_cols = 1.0f / (float)q.cols, c1 = sum[0] * over_cols;
    return make_float2(c1, q.post_norm ? (sum[1] - rs * c1 * sum[2]) * over_cols : 0.0f);
}

// The means of rows that are wider than a workgroup; k_block_norm_backward then takes such rows in strips.  The operands are read twice: 4096 x 16384 from
// 8-bit checkpoints takes 242 to 251 us in all (4.4 TB/s of what is moved).  With two pieces per lane in one kernel the sums over rows did not fit the registers: 445 us.
template <bool KEPT, bool SF32, bool YF32> __global__ __launch_bounds__(ROW_THREADS) void k_block_norm_means(adahop_block_norm_t q, float2 *means)
{
    __shared__ row_sums_t<3> lds;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < q.rows; row += gridDim.x) {
        const int64_t gate_row = q.gate.data ? row / q.gate_rows : 0;
        const float rs = q.d_h.data ? q.rstd_pre[row] : 0.0f, ry = q.post_norm ? q.rstd_post[row] : 1.0f;
        float sum[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll 1
        for (int c = threadIdx.x * 8; c < (int)q.cols; c += 8 * ROW_THREADS) {
            const int n = (int)q.cols - c;
            constexpr bool ODD = true;
            piece_t<ODD, KEPT, SF32, YF32> p;
            float wpre[8], wbranch[8];
            p.load(q, row, c, n);
            vector_of<ODD>(q.w_pre, c, n, wpre);
            branch_of<ODD>(q, gate_row, c, n, wbranch);
            p.add(n, rs, ry, wpre, wbranch, sum);
        }
        row_sums(lds, turn, ROW_THREADS / 64, sum);
        if (threadIdx.x == 0) means[row] = means_of(q, rs, sum);
    }
}

// BESIDE: several runs per workgroup; STRIPS: rows wider than a workgroup, whose means are there already: blockIdx.y is the strip; ODD: a row's last piece may
// be a part (whole pieces without the paths for a part: 8192 x 4096 with token gates and checkpoints 109 us instead of
// 124, 8192 x 2048 67 instead of 75); SF32: ds, dx
// and a saved s are fp32; YF32: dh, dy and a saved y are.
//
// One accumulator serves both the gate and w_post: with A = sum(beta d yhat) over rows of one gate row, its gate gradient is w_post A and its part of
// w_post's is gate A.  CUT: all rows of the run are of one gate row.  The row's values stay as they were loaded over the barrier and are widened again behind it
// (half the registers).  The next row is loaded meanwhile where a row takes few registers as it lies in memory (RAW), a rule on types alone: 8192 x 4096 with token gates,
// the stream in fp32 and 8-bit checkpoints, took 174 us with the next row, 140 without.  It leaves spills: from checkpoints under CUT, with the stream or the
// block's side in fp32, 2 to 10 of the 128 registers (16384 x 8192 with the stream in fp32 takes 379 us, 5.0 TB/s, all the same); up to 3 elsewhere with a row ahead, up to 10
// without one where everything is fp32.
template <bool BESIDE, bool STRIPS, bool ODD, bool KEPT, bool CUT, bool SF32, bool YF32> __global__ __launch_bounds__(ROW_THREADS) void k_block_norm_backward(backward_t b)
{
    // registers that a row takes as it lies in memory: two rows at a time where that leaves enough for the rest
    constexpr int RAW = (SF32 ? 8 : 4) + (YF32 ? 8 : 4) + (KEPT ? 6 : (SF32 ? 8 : 4) + (YF32 ? 8 : 4));
    constexpr bool AHEAD = RAW <= (CUT ? 22 : 16);
    __shared__ row_sums_t<3> lds;
    __shared__ float patch[BESIDE ? 8 * ROW_THREADS : 1];
    const adahop_block_norm_t &q = b.q;
    const int threads = BESIDE ? b.threads : blockDim.x, waves = threads >> 6, sub = BESIDE ? __builtin_amdgcn_readfirstlane(threadIdx.x / threads) : 0;
    const int tid = threadIdx.x - sub * threads, col = (STRIPS ? blockIdx.y * threads + tid : tid) * 8, left = (int)q.cols - col;
    int turn = 0;
    float wbranch[8], wpre[8], apre[8], apost[8], agate[8]; // agate: A of the gate row at hand
#pragma unroll
    for (int i = 0; i < 8; ++i) apre[i] = apost[i] = agate[i] = 0.0f;
    vector_of<ODD>(q.w_pre, col, left, wpre);
    const int64_t run = BESIDE ? (int64_t)blockIdx.x * b.runs.beside + sub : blockIdx.x;
    int64_t row = run * b.runs.rows, end = row + b.runs.rows;
    if constexpr (CUT) {
        const int64_t g = run / b.runs.cuts, cut = run % b.runs.cuts;
        row = g * b.runs.group + cut * b.runs.rows;
        end = row + b.runs.rows < (g + 1) * b.runs.group ? row + b.runs.rows : (g + 1) * b.runs.group;
    }
    if (end > q.rows) end = q.rows;
    const bool any = row < end; // or there is no such run
    const int64_t fewer = b.runs.rows - (any ? end - row : 0); // rows than other runs of the workgroup may have
    piece_t<ODD, KEPT, SF32, YF32> next;
    float rs = 0.0f, ry = 1.0f;
    const auto load_row = [&](int64_t r) {
        if (q.d_h.data) rs = q.rstd_pre[r];
        if (q.post_norm) ry = q.rstd_post[r];
        next.load(q, r, col, left);
    };
    int64_t gate_row = 0, gate_until = row; // first row of another gate row than the present one
    if (row < end) load_row(row);
    while (row < end) {
        if (row >= gate_until) {
            gate_row = q.gate.data ? row / q.gate_rows : 0;
            gate_until = q.gate.data ? (gate_row + 1) * q.gate_rows : end;
            branch_of<ODD>(q, gate_row, col, left, wbranch);
        }
        float sum[3] = {0.0f, 0.0f, 0.0f};
        if constexpr (!STRIPS) next.add(left, rs, ry, wpre, wbranch, sum);
        piece_t<ODD, KEPT, SF32, YF32> at = next;
        keep_raw(at.ds), keep_raw(at.dh), keep_raw(at.s.r), keep_raw(at.y.r);
        const float rs0 = rs, ry0 = ry;
        if constexpr (AHEAD) {
            if (row + 1 < end) load_row(row + 1);
        }
        float2 mean;
        if constexpr (STRIPS) {
            mean = b.means[row];
        } else {
            row_sums(lds, turn, waves, sum, sub * waves);
            mean = means_of(q, rs0, sum);
        }
        float d[8], t[8], shat[8], yhat[8], dx[8], dy[8];
        widen8(at.ds, d);
        widen8(at.dh, t);
        widen_saved(at.s, rs0, shat);
        widen_saved(at.y, ry0, yhat);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            apre[i] = __builtin_fmaf(t[i], shat[i], apre[i]);
            d[i] = __builtin_fmaf(rs0, __builtin_fmaf(-mean.x, shat[i], t[i] * wpre[i]), d[i]);
            dx[i] = q.residual_scale * d[i];
            dy[i] = ry0 * __builtin_fmaf(-mean.y, yhat[i], d[i] * wbranch[i]);
            agate[i] = __builtin_fmaf(q.branch_scale * d[i], yhat[i], agate[i]);
        }
        if (left > 0) {
            if (q.d_x.data) store8<SF32, ODD>(q.d_x.data, row * q.d_x.ld + col, left, dx);
            if (q.d_y.data) store8<YF32, ODD>(q.d_y.data, row * q.d_y.ld + col, left, dy);
        }
        ++row;
        if constexpr (!CUT) {
            if (row == end || row == gate_until) { // the gate row is complete
                float g[8], w[8];
                vector_of<ODD>(q.gate, gate_row * q.gate.ld + col, to_load(left, gate_row + 1 < q.gates, q.cols), g);
                vector_of<ODD>(q.w_post, col, left, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    apost[i] = __builtin_fmaf(agate[i], g[i], apost[i]);
                    w[i] *= agate[i];
                    agate[i] = 0.0f;
                }
                if (q.d_gate.data && left > 0) store8_any<ODD>(q.d_gate, gate_row * q.d_gate.ld + col, left, w);
            }
        }
        if constexpr (!AHEAD) {
            if (row < end) load_row(row);
        }
    }
    if (BESIDE && waves > 1) // the barriers of their sums
        for (int64_t i = 0; i < fewer; ++i) __syncthreads();
    // One gradient's part, as it is or the runs' sum, to fp32 row `to`.
    const auto hand_over = [&](const float (&v)[8], float *to) {
        if constexpr (!BESIDE) {
            if (left > 0) store8<true, ODD>(to, col, left, v);
        } else {
            __syncthreads(); // no wave reads the one before any more
            float4 *const mine = reinterpret_cast<float4 *>(patch + 8 * threadIdx.x);
            mine[0] = make_float4(v[0], v[1], v[2], v[3]);
            mine[1] = make_float4(v[4], v[5], v[6], v[7]);
            __syncthreads();
            for (int c = threadIdx.x; c < (int)q.cols; c += blockDim.x) {
                float sum = patch[c];
                for (int k = 1; k < b.runs.beside; ++k) sum += patch[8 * threads * k + c];
                to[c] = sum;
            }
        }
    };
    float *const part = b.part ? b.part + blockIdx.x * q.cols : nullptr;
    const int64_t one = b.workgroups * q.cols;
    if (q.d_w_pre) hand_over(apre, part ? part : q.d_w_pre);
    if constexpr (CUT) {
        float v[8];
        if (q.d_gate.data) {
            vector_of<ODD>(q.w_post, col, left, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = any ? v[i] * agate[i] : 0.0f;
            if (!BESIDE || b.runs.joined)
                hand_over(v, part + 2 * one); // (a single row is no part of a group)
            else if (run < b.runs.number && left > 0)
                store8<true, ODD>(b.part + 2 * one, run * q.cols + col, left, v);
        }
        vector_of<ODD>(q.gate, gate_row * q.gate.ld + col, left, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) apost[i] = any ? v[i] * agate[i] : 0.0f;
    }
    if (q.d_w_post) hand_over(apost, part ? part + one : q.d_w_post);
}

// Sums of the workgroups' parts.  blockIdx.y = 0, 1: the weight gradients; from 2 on the gate rows.  A workgroup takes 64 columns; its waves
// share the parts, each in order, and their sums are added in order.  Bound by the way to memory and back: a thread's loads are on their way BATCH
// at a time, the last ones too (256 parts of 8192 columns, three sums: 5.3 us).
constexpr int REDUCE_THREADS = 1024, BATCH = 16;

__global__ __launch_bounds__(REDUCE_THREADS) void k_block_norm_reduce(backward_t b)
{
    constexpr int WAVES = REDUCE_THREADS / 64;
    __shared__ float lds[WAVES][64];
    const int which = blockIdx.y < 2 ? blockIdx.y : 2;
    float *const to = which == 0 ? b.q.d_w_pre : which == 1 ? b.q.d_w_post : nullptr;
    if (which < 2 ? !to : !b.q.d_gate.data) return; // of the whole workgroup
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane, first = which < 2 ? 0 : (int64_t)(blockIdx.y - 2) * b.gate_cuts;
    const int64_t parts = which < 2 ? b.workgroups : b.gate_cuts, share = (parts + WAVES - 1) / WAVES;
    const int64_t begin = w * share, end = begin + share < parts ? begin + share : parts;
    float sum = 0.0f;
    if (c < b.q.cols) {
        const float *p = b.part + (which * b.workgroups + first + begin) * b.q.cols + c;
        for (int64_t i = begin; i < end; i += BATCH, p += BATCH * b.q.cols) {
            float v[BATCH]; // where fewer are left, the first again
#pragma unroll
            for (int j = 0; j < BATCH; ++j) v[j] = p[(i + j < end ? j : 0) * b.q.cols];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) sum += i + j < end ? v[j] : 0.0f;
        }
    }
    lds[w][lane] = sum;
    __syncthreads();
    if (w || c >= b.q.cols) return;
#pragma unroll
    for (int i = 1; i < WAVES; ++i) sum += lds[i][lane];
    if (which < 2)
        to[c] = sum;
    else
        put(b.q.d_gate, (int64_t)(blockIdx.y - 2) * b.q.d_gate.ld + c, sum);
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
    for (int64_t g = from + blockIdx.y; g < q.gates; g += gridDim.y) put(q.d_gate, g * q.d_gate.ld + c, 0.0f);
}

int zero_gates_from(const adahop_block_norm_t &q, int64_t from, hipStream_t st)
{
    const int64_t gates = q.d_gate.data ? q.gates - from : 0;
    k_block_norm_zero<<<dim3((unsigned)ceil_div(q.cols, 256), (unsigned)(gates < 1 ? 1 : gates > 1024 ? 1024 : gates)), 256, 0, st>>>(q, from);
    return check_launch();
}

template <bool BESIDE, bool STRIPS, bool ODD, bool KEPT, bool CUT> void launch(const backward_t &b, bool s32, bool y32, hipStream_t st)
{
    const dim3 n((unsigned)b.workgroups, (unsigned)strips_of(b.q.cols));
    const unsigned threads = b.threads * b.runs.beside;
    if (s32)
        y32 ? k_block_norm_backward<BESIDE, STRIPS, ODD, KEPT, CUT, true, true><<<n, threads, 0, st>>>(b)
            : k_block_norm_backward<BESIDE, STRIPS, ODD, KEPT, CUT, true, false><<<n, threads, 0, st>>>(b);
    else
        y32 ? k_block_norm_backward<BESIDE, STRIPS, ODD, KEPT, CUT, false, true><<<n, threads, 0, st>>>(b)
            : k_block_norm_backward<BESIDE, STRIPS, ODD, KEPT, CUT, false, false><<<n, threads, 0, st>>>(b);
}

template <bool BESIDE, bool STRIPS, bool ODD> void launch(const backward_t &b, bool s32, bool y32, bool kept, hipStream_t st)
{
    if (kept)
        b.runs.cuts ? launch<BESIDE, STRIPS, ODD, true, true>(b, s32, y32, st) : launch<BESIDE, STRIPS, ODD, true, false>(b, s32, y32, st);
    else
        b.runs.cuts ? launch<BESIDE, STRIPS, ODD, false, true>(b, s32, y32, st) : launch<BESIDE, STRIPS, ODD, false, false>(b, s32, y32, st);
}

template <bool KEPT> void launch_means(const adahop_block_norm_t &q, float2 *means, bool s32, bool y32, hipStream_t st)
{
    const unsigned n = (unsigned)(q.rows < 8 * COMPUTE_UNITS ? q.rows : 8 * COMPUTE_UNITS);
    if (s32)
        y32 ? k_block_norm_means<KEPT, true, true><<<n, ROW_THREADS, 0, st>>>(q, means) : k_block_norm_means<KEPT, true, false><<<n, ROW_THREADS, 0, st>>>(q, means);
    else
        y32 ? k_block_norm_means<KEPT, false, true><<<n, ROW_THREADS, 0, st>>>(q, means) : k_block_norm_means<KEPT, false, false><<<n, ROW_THREADS, 0, st>>>(q, means);
}

size_t means_bytes(int64_t rows, int64_t cols) { return strips_of(cols) > 1 ? align_up((size_t)rows * sizeof(float2), 256) : 0; }

} // namespace

size_t block_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t gate_rows)
{
    if (rows == 0) return 0;
    const runs_t r = runs_of(rows, cols, gate_rows);
    return means_bytes(rows, cols) + (rows == 1 ? 0 : (size_t)(2 * r.workgroups() + r.gate_parts()) * cols * sizeof(float));
}

int launch_block_norm_no_rows(const adahop_block_norm_t &q, hipStream_t st) { return zero_gates_from(q, 0, st); }

int launch_block_norm_backward(const adahop_block_norm_t &q, bool s32, bool y32, bool kept, void *workspace, hipStream_t st)
{
    const runs_t r = runs_of(q.rows, q.cols, q.gate.data ? q.gate_rows : 0);
    float2 *const means = strips_of(q.cols) > 1 ? static_cast<float2 *>(workspace) : nullptr;
    float *const part = q.rows == 1 ? nullptr : reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + means_bytes(q.rows, q.cols));
    const backward_t b = {q, r, threads_of(q.cols), r.gate_cuts(), r.workgroups(), means, part};
    if (means) {
        kept ? launch_means<true>(q, means, s32, y32, st) : launch_means<false>(q, means, s32, y32, st);
        const int rc = check_launch();
        if (rc != ADAHOP_OK) return rc;
        launch<false, true, true>(b, s32, y32, kept, st);
    } else if (r.beside > 1) {
        q.cols % 8 ? launch<true, false, true>(b, s32, y32, kept, st) : launch<true, false, false>(b, s32, y32, kept, st);
    } else {
        q.cols % 8 ? launch<false, false, true>(b, s32, y32, kept, st) : launch<false, false, false>(b, s32, y32, kept, st);
    }
    int rc = check_launch();
    if (rc == ADAHOP_OK && q.d_gate.data && q.gates > ceil_div(q.rows, q.gate_rows)) rc = zero_gates_from(q, ceil_div(q.rows, q.gate_rows), st);
    if (rc != ADAHOP_OK || !b.part) return rc;
    const int64_t gates = q.d_gate.data && b.runs.cuts ? ceil_div(q.rows, b.runs.group) : 0;
    if (!q.d_w_pre && !q.d_w_post && !gates) return ADAHOP_OK;
    k_block_norm_reduce<<<dim3((unsigned)ceil_div(q.cols, 64), (unsigned)(2 + gates)), REDUCE_THREADS, 0, st>>>(b);
    return check_launch();
}

} // namespace adahop

// The norms after one block and before the next, with what stands between them (forward):
//
//     yhat = y / sqrt(mean(y^2) + eps),   s = alpha x + beta gate * w_post * yhat
//     shat = s / sqrt(mean(s^2) + eps),   h = w_pre * shat
//
// in one pass: a workgroup holds a row in registers, eight consecutive elements per lane and piece, and sums its squares
// twice.  Bound by the memory: x and y are read once, s, h and the 8-bit checkpoints of yhat and shat are written once; for a single row of 4096 by
// its latency, 4.5 us of which some 2 are the launch.  The sums are in fp32; h and the checkpoints are formed from s before its rounding to bf16,
// so that each output is rounded once.
#include "ckpt8.h"
#include "row_sums.h"

namespace adahop {

namespace {

// 1 / sqrt(m), the nearest number or, seldom, the one beside it: the nearest root's nearest reciprocal, and one Newton step from it, whose
// remainder 1 - m r^2 is formed without rounding m r.  Without that step the factor is off by 4.4e-8 instead of 3.4e-8 (rms, the sum's share
// included), and more codes of a row's checkpoint lie on the other side of a tie.
__device__ __forceinline__ float over_root(float m)
{
    const float r = 1.0f / sqrtf(m), p = m * r;
    const float e = __builtin_fmaf(-__builtin_fmaf(m, r, -p), r, __builtin_fmaf(-p, r, 1.0f));
    return fabsf(e) < 1.0f ? __builtin_fmaf(0.5f * r, e, r) : r; // of an infinity 0, of NaN NaN
}

// C: pieces of 8 columns per lane; ODD: the last one may be a part; SF32, YF32: the type of x and s, and of y.  The next
// row's x and y are on their way while a row is summed.  Rows of whole pieces have kernels of their own, without the
// paths for a part: 8192 x 4096 in 52.1 us instead of 57.8, 16384 x 8192 with both checkpoints in 246 us instead of
// 259 (239 us, 5.65 TB/s, at best).
template <int C, bool ODD, bool SF32, bool YF32> __global__ __launch_bounds__(ROW_THREADS) void k_block_norm(adahop_block_norm_t q)
{
    __shared__ row_sums_t<1> lds;
    const int threads = blockDim.x, waves = threads >> 6;
    int turn = 0;
    const auto col = [&](int j) { return (int)(threadIdx.x + j * threads) * 8; };
    const auto left = [&](int j) { return (int)q.cols - col(j); };
    float wbranch[C][8], wpre[C][8]; // branch_scale w_post gate; w_pre
#pragma unroll
    for (int j = 0; j < C; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) wpre[j][i] = wbranch[j][i] = 1.0f;
        if (q.w_pre.data && left(j) > 0) load8_any<ODD>(q.w_pre, col(j), left(j), wpre[j]);
    }
    raw8<SF32> x[C];
    raw8<YF32> y[C];
    const auto load_row = [&](int64_t row) {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const int n = to_load(left(j), row + 1 < q.rows, q.cols);
            x[j] = q.x.data && n > 0 ? load8<SF32, ODD>(q.x.data, row * q.x.ld + col(j), n) : zero8<SF32>();
            y[j] = q.y.data && n > 0 ? load8<YF32, ODD>(q.y.data, row * q.y.ld + col(j), n) : zero8<YF32>();
        }
    };
    const float over = 1.0f / (float)q.cols, rest = __builtin_fmaf(-over, (float)q.cols, 1.0f) * over; // together 1 / cols
    // An infinite sum (an infinity in the row, or squares past fp32) takes part in the larger of the two products alone: `rest` is 0 or negative at most widths.
    const auto rstd = [&](float squares) { return over_root(__builtin_fmaf(squares, over, squares < INFINITY ? __builtin_fmaf(squares, rest, q.eps) : q.eps)); };
    const float alpha = q.x.data ? q.residual_scale : 0.0f;
    int64_t gate_until = 0; // first row of another gate row than the present one
    if (blockIdx.x < q.rows) load_row(blockIdx.x);
    for (int64_t row = blockIdx.x; row < q.rows; row += gridDim.x) {
        float z[C][8], v[C][8], sum[1];
        if (row >= gate_until) {
            const int64_t gate_row = q.gate.data ? row / q.gate_rows : 0;
            gate_until = q.gate.data ? (gate_row + 1) * q.gate_rows : q.rows;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                float g[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f}, w[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
                const int n = to_load(left(j), gate_row + 1 < q.gates, q.cols);
                if (q.gate.data && n > 0) load8_any<ODD>(q.gate, gate_row * q.gate.ld + col(j), n, g);
                if (q.w_post.data && left(j) > 0) load8_any<ODD>(q.w_post, col(j), left(j), w);
#pragma unroll
                for (int i = 0; i < 8; ++i) wbranch[j][i] = q.branch_scale * w[i] * g[i];
            }
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            widen8(x[j], z[j]);
            widen8(y[j], v[j]);
            if (ODD && left(j) < 8) zero_from(left(j), v[j]);
        }
        if (row + gridDim.x < q.rows) load_row(row + gridDim.x);
        if (q.post_norm) {
            sum[0] = 0.0f;
#pragma unroll
            for (int j = 0; j < C; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] = __builtin_fmaf(v[j][i], v[j][i], sum[0]);
            row_sums(lds, turn, waves, sum);
            const float r = rstd(sum[0]);
            if (q.rstd_post && threadIdx.x == 0) q.rstd_post[row] = r;
#pragma unroll
            for (int j = 0; j < C; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] *= r;
        }
        if (q.ckpt_y.codes) {
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const packed8 k = pack8(v[j]);
                if (left(j) > 0) store_packed8<ODD>(q.ckpt_y, row, col(j), left(j), k);
            }
        }
        sum[0] = 0.0f;
#pragma unroll
        for (int j = 0; j < C; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[j][i] = alpha * z[j][i] + v[j][i] * wbranch[j][i];
            if (ODD && left(j) < 8) zero_from(left(j), z[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] = __builtin_fmaf(z[j][i], z[j][i], sum[0]);
            if (q.s.data && left(j) > 0) store8<SF32, ODD>(q.s.data, row * q.s.ld + col(j), left(j), z[j]);
        }
        if (!q.h.data) continue;
        row_sums(lds, turn, waves, sum);
        const float r = rstd(sum[0]);
        if (q.rstd_pre && threadIdx.x == 0) q.rstd_pre[row] = r;
#pragma unroll
        for (int j = 0; j < C; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[j][i] *= r;
            if (q.ckpt_s.codes) {
                const packed8 k = pack8(z[j]);
                if (left(j) > 0) store_packed8<ODD>(q.ckpt_s, row, col(j), left(j), k);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) z[j][i] *= wpre[j][i];
            if (left(j) > 0) store8_any<ODD>(q.h, row * q.h.ld + col(j), left(j), z[j]);
        }
    }
}

template <int C, bool ODD> void launch(const adahop_block_norm_t &q, int threads, unsigned groups, hipStream_t st)
{
    if (q.s.data ? q.s.f32 : q.x.f32)
        q.y.f32 ? k_block_norm<C, ODD, true, true><<<groups, threads, 0, st>>>(q) : k_block_norm<C, ODD, true, false><<<groups, threads, 0, st>>>(q);
    else
        q.y.f32 ? k_block_norm<C, ODD, false, true><<<groups, threads, 0, st>>>(q) : k_block_norm<C, ODD, false, false><<<groups, threads, 0, st>>>(q);
}

} // namespace

int launch_block_norm(const adahop_block_norm_t &q, hipStream_t st)
{
    const int64_t pieces = ceil_div(q.cols, 8);
    const int threads = (int)(pieces > ROW_THREADS ? ROW_THREADS : ceil_div(pieces, 64) * 64);
    const int64_t most = 256 * (int64_t)(2048 / threads); // 256 compute units of 2048 threads at most
    const unsigned groups = (unsigned)(q.rows < most ? q.rows : most);
    if (pieces > ROW_THREADS)
        launch<2, true>(q, threads, groups, st);
    else
        q.cols % 8 ? launch<1, true>(q, threads, groups, st) : launch<1, false>(q, threads, groups, st);
    return check_launch();
}

} // namespace adahop

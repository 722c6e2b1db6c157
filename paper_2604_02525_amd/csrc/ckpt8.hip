// 8-bit activation checkpoints (packing, unpacking) and the gated activation a = silu(g) u that writes and reads them.
// All four are elementwise but for the scale of 32 features: bound by the memory, one pass over it.  A lane has one piece of 8 elements (16-byte
// accesses in bf16), four neighbouring lanes have a block of 32 and find its largest magnitude by two lane exchanges.  One piece per lane and very many
// workgroups, not a loop: the hardware keeps the loads of thousands of waves on their way by itself.
#include "ckpt8.h"

namespace adahop {

namespace {

// The lane's piece: its row, its first column, and how many of its 8 elements exist (none: <= 0).
struct piece_t {
    uint32_t row;
    int c, n;
};

// Blocks are numbered, not pieces: up to 2^30 + 2^21 blocks there may be, four times as many pieces pass 32 bits.
__device__ __forceinline__ piece_t piece_of(const blocks_t &g, int cols)
{
    const uint32_t at = (blockIdx.y * g.across + blockIdx.x) * (PIECES / 4) + (threadIdx.x >> 2);
    piece_t p;
    uint32_t b;
    block_at(g, at, &p.row, &b);
    p.c = (int)(b * 32 + (threadIdx.x & 3) * 8);
    p.n = at < g.total ? cols - p.c : 0;
    return p;
}

// 8192 x 4096 bf16: 17.4 us, 5.8 TB/s (the input of 67 MB lies in the 256 MB cache).
template <bool F32> __global__ __launch_bounds__(PIECES) void k_ckpt8_pack(adahop_tensor_t x, adahop_ckpt8_t out, blocks_t g, int cols)
{
    const piece_t p = piece_of(g, cols);
    float v[8];
    widen8(p.n > 0 ? load8<F32>(x.data, p.row * x.ld + p.c, p.n) : zero8<F32>(), v);
    const packed8 k = pack8(v);
    if (p.n > 0) store_packed8(out, p.row, p.c, p.n, k);
}

// 16384 x 8192 to bf16: 68.8 us, 5.9 TB/s.
template <bool F32> __global__ __launch_bounds__(PIECES) void k_ckpt8_unpack(adahop_ckpt8_t x, adahop_tensor_t scale, adahop_tensor_t out, blocks_t g, int cols)
{
    const piece_t p = piece_of(g, cols);
    if (p.n <= 0) return;
    float v[8];
    unpack8(load_packed8(x, p.row, p.c, p.n), v);
    if (scale.data) {
        float w[8];
        load8_any(scale, p.c, p.n, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= w[i];
    }
    store8<F32>(out.data, p.row * out.ld + p.c, p.n, v);
}

// The exponential and the reciprocal as the hardware has them.  exp(-g) is 2 to the power of -g log2(e), a product rounded to fp32, so the result is off by up to
// (2 |g| + 16) 2^-24 of itself: far below the rounding to bf16 or to 8 bits that follows (2^-9 and 2^-4) wherever the result counts; of outputs in fp32 the
// last five to seven bits at |g| of 10 to 60.
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

// 8192 x 11008 bf16 with both checkpoints: 122.5 us, 5.9 TB/s (127 before the codes went past the caches).
template <bool F32> __global__ __launch_bounds__(PIECES) void k_swiglu(adahop_swiglu_t q, blocks_t b, int cols)
{
    const piece_t p = piece_of(b, cols);
    float g[8], u[8], a[8];
    widen8(p.n > 0 ? load8<F32>(q.g.data, p.row * q.g.ld + p.c, p.n) : zero8<F32>(), g);
    widen8(p.n > 0 ? load8<F32>(q.u.data, p.row * q.u.ld + p.c, p.n) : zero8<F32>(), u);
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = g[i] * sigmoid(g[i]) * u[i];
    if (p.n > 0) store8_any(q.a, p.row * q.a.ld + p.c, p.n, a);
    if (q.ckpt_g.codes) {
        const packed8 k = pack8(g);
        if (p.n > 0) store_packed8(q.ckpt_g, p.row, p.c, p.n, k);
    }
    if (q.ckpt_u.codes) {
        const packed8 k = pack8(u);
        if (p.n > 0) store_packed8(q.ckpt_u, p.row, p.c, p.n, k);
    }
}

// silu'(g) = sigma + g sigma (1 - sigma).  8192 x 11008 from both checkpoints, a handed back in 8 bits: 137 us, 6.0 TB/s; 301 x 14333 from bf16, the gradient in
// fp32: 12.6 us, 4.8 TB/s (no row but the first begins at a multiple of 16 bytes).
template <bool KEPT, bool F32> __global__ __launch_bounds__(PIECES) void k_swiglu_backward(adahop_swiglu_t q, blocks_t b, int cols)
{
    const piece_t p = piece_of(b, cols);
    float g[8] = {}, u[8] = {}, da[8], dg[8], du[8], a[8];
    widen8(p.n > 0 ? load8<F32>(q.d_a.data, p.row * q.d_a.ld + p.c, p.n) : zero8<F32>(), da);
    if (p.n > 0) {
        if constexpr (KEPT) {
            const packed8 kg = load_packed8(q.ckpt_g, p.row, p.c, p.n), ku = load_packed8(q.ckpt_u, p.row, p.c, p.n);
            unpack8(kg, g);
            unpack8(ku, u);
        } else {
            load8_any(q.g, p.row * q.g.ld + p.c, p.n, g);
            load8_any(q.u, p.row * q.u.ld + p.c, p.n, u);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = sigmoid(g[i]), silu = g[i] * s;
        a[i] = silu * u[i];
        du[i] = da[i] * silu;
        dg[i] = da[i] * u[i] * (s + silu * (1.0f - s));
    }
    if (p.n > 0) {
        store8_any(q.d_g, p.row * q.d_g.ld + p.c, p.n, dg);
        store8_any(q.d_u, p.row * q.d_u.ld + p.c, p.n, du);
        if (q.a.data) store8_any(q.a, p.row * q.a.ld + p.c, p.n, a);
    }
    if (q.ckpt_a.codes) {
        const packed8 k = pack8(a);
        if (p.n > 0) store_packed8(q.ckpt_a, p.row, p.c, p.n, k);
    }
}

inline dim3 groups_of(const blocks_t &g) { return dim3(g.across, (unsigned)ceil_div(ceil_div((int64_t)g.total * 4, PIECES), g.across)); }

} // namespace

int launch_ckpt8_pack(int64_t rows, int64_t cols, const adahop_tensor_t &x, const adahop_ckpt8_t &out, hipStream_t st)
{
    const blocks_t g = blocks_of(rows, cols);
    if (x.f32)
        k_ckpt8_pack<true><<<groups_of(g), PIECES, 0, st>>>(x, out, g, (int)cols);
    else
        k_ckpt8_pack<false><<<groups_of(g), PIECES, 0, st>>>(x, out, g, (int)cols);
    return check_launch();
}

int launch_ckpt8_unpack(int64_t rows, int64_t cols, const adahop_ckpt8_t &x, const adahop_tensor_t &scale, const adahop_tensor_t &out, hipStream_t st)
{
    const blocks_t g = blocks_of(rows, cols);
    if (out.f32)
        k_ckpt8_unpack<true><<<groups_of(g), PIECES, 0, st>>>(x, scale, out, g, (int)cols);
    else
        k_ckpt8_unpack<false><<<groups_of(g), PIECES, 0, st>>>(x, scale, out, g, (int)cols);
    return check_launch();
}

int launch_swiglu(const adahop_swiglu_t &q, hipStream_t st)
{
    const blocks_t g = blocks_of(q.rows, q.cols);
    if (q.g.f32)
        k_swiglu<true><<<groups_of(g), PIECES, 0, st>>>(q, g, (int)q.cols);
    else
        k_swiglu<false><<<groups_of(g), PIECES, 0, st>>>(q, g, (int)q.cols);
    return check_launch();
}

int launch_swiglu_backward(const adahop_swiglu_t &q, hipStream_t st)
{
    const blocks_t g = blocks_of(q.rows, q.cols);
    const dim3 n = groups_of(g);
    const int cols = (int)q.cols;
    if (q.ckpt_g.codes)
        q.d_a.f32 ? k_swiglu_backward<true, true><<<n, PIECES, 0, st>>>(q, g, cols) : k_swiglu_backward<true, false><<<n, PIECES, 0, st>>>(q, g, cols);
    else
        q.d_a.f32 ? k_swiglu_backward<false, true><<<n, PIECES, 0, st>>>(q, g, cols) : k_swiglu_backward<false, false><<<n, PIECES, 0, st>>>(q, g, cols);
    return check_launch();
}

} // namespace adahop

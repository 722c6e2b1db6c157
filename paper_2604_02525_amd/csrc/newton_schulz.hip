// Orthogonalisation of a matrix by Newton-Schulz products, and the update of a weight by it:
//
//     X = U / (|U| + eps),   repeat `steps` times:  A = X X^T,  X <- a X + (b A + c A^2) X,   out = scale X
//
// (for a matrix of more rows than columns A = X^T X, from the other side).  U is the matrix given, or for an update of a weight its gradient with momentum:
// m' = mu m + g, U = g + mu m' (nesterov) or m', w' = (1 - rate decay) w - rate scale X.
//
// The singular values of X pass through a x + b x^3 + c x^5 in every step, and with them what rounding adds: directions that are weak at first grow by a factor of a.
// Plain 16-bit iterates lose them (bf16: 1 to 15 % of the result).  What this does instead, each product still being one pass of 16-bit operands:
//   * X is carried in fp32; only what enters the products is rounded, to fp16 (times a power of two), so that a X is exact.
//   * The diagonals of A and of b A + c A^2 are apart, in fp32: they are by far the largest elements, their rounding would be the largest error.  With A = D + O:
//     the polynomial is b (D + O) + c (D^2 + D O + O D + O^2), of which the matrix cores form O^2, and its diagonal joins a in what multiplies the carried X.
//   * Where the smaller side is at most 128, X enters as the sum of two fp16 numbers: errors there average over fewer elements, and the products cost little.
//   * In the steps whose noise later ones multiply, the diagonal takes X as the products take it (as_rounded_t).
// The result of five steps is then 2e-4 to 1.2e-3 of its norm off the same iteration in 64 bits for matrices of random elements and gradients with a few strong directions (bf16's own rounding: 1.7e-3), 4e-3 at most
// whatever the singular values, 5e-3 where the elements are two or four different numbers; in ten steps 3e-3 and 1.2e-2 (one direction alone: the fp32 iterate's rounding times 3.4445^10).
//
// A and A^2 are symmetric: only tiles on and below the diagonal are computed, the mirror image is stored with them.  (Within a tile on the diagonal of an A of two numbers the two halves are sums
// in another order, equal to rounding.)
//
// What bounds it (five steps): large matrices the matrix cores' power, and the step product's end, which reads and writes 10 bytes an element of fp32 and fp16 iterates (28672 x 8192 updated: 28.1 to 28.8 ms on different cards,
// 1.10 to 1.12 PFLOP/s of what is counted once); middle ones rounds of tiles that do not fill the card (4096 x 4096: 1.42 to 1.47 ms, 0.94 to 0.97; 2048 x 2048 updated: 0.35 to 0.37 ms, 0.47 to 0.49), where the split of the last round into slices and the choice of tiles is
// worth most; small ones 17 launches of some 5 us that wait for each other (256 x 256: 87 us, 185 with tiles of 128 or more).
#include <math.h>

#include "tile16.h"

namespace adahop {

namespace {

constexpr int SX = 12, SO = 12, SB = 10; // X, O and the polynomial's off-diagonal part are held times 2^S in fp16: below 16, 16 and 64
constexpr int PARTS = 1024;              // workgroups of the sum of squares, at most
constexpr int SPLIT_SIDE = 128;

constexpr float pow2(int e) { return e >= 0 ? (float)((uint64_t)1 << e) : 1.0f / (float)((uint64_t)1 << -e); }

__device__ __forceinline__ uint32_t f16_pair(float a, float b) // round to nearest even
{
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    const v2h p = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ u32x2 f16_four(const float (&v)[4]) { return u32x2{f16_pair(v[0], v[1]), f16_pair(v[2], v[3])}; }
__device__ __forceinline__ void f16_values(u32x2 w, float (&v)[4])
{
    typedef _Float16 v4h __attribute__((ext_vector_type(4)));
    const v4h h = __builtin_bit_cast(v4h, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)h[i];
}
__device__ __forceinline__ void store_eight(uint16_t *to, const float (&v)[8])
{
    *reinterpret_cast<u32x4 *>(to) = u32x4{f16_pair(v[0], v[1]), f16_pair(v[2], v[3]), f16_pair(v[4], v[5]), f16_pair(v[6], v[7])};
}

// ---- before the products ----------------------------------------------------------------------------------------------------------
struct source_t {
    adahop_tensor_t g, m, m_out; // m, m_out: absent without momentum
    float mu;
    int nesterov;
    int64_t rows, cols;
};

// n <= 8 elements of U from (r, c) on, zeros behind them; with momentum from what it has become.
__device__ __forceinline__ void u_at(const source_t &s, const adahop_tensor_t &m, int64_t r, int64_t c, int n, bool advance, float (&u)[8])
{
    load8_any(s.g, r * s.g.ld + c, n, u);
    if (!m.data) return;
    float v[8];
    load8_any(m, r * m.ld + c, n, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (advance) v[i] = s.mu * v[i] + u[i];
        u[i] = s.nesterov ? u[i] + s.mu * v[i] : v[i];
    }
    if (advance) store8_any(s.m_out, r * s.m_out.ld + c, n, v);
}

// The momentum's step, and sums of U's squares, in 64 bits: no element is too large or too small for them.
__global__ __launch_bounds__(256) void k_squares(source_t s, double *part)
{
    __shared__ double of_wave[4];
    const int64_t pieces = (s.cols + 7) / 8, all = s.rows * pieces;
    double sum = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces, c = (i - r * pieces) * 8;
        float u[8];
        u_at(s, s.m, r, c, (int)(s.cols - c < 8 ? s.cols - c : 8), true, u);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += (double)u[k] * u[k];
    }
#pragma unroll
    for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = of_wave[0] + of_wave[1] + of_wave[2] + of_wave[3];
}

// Where the iterates are held: [rows_pad][ld], both multiples of 64, zeros outside the matrix.
struct iterate_t {
    float *x;
    uint16_t *h; // fp16 of x 2^SX; split: what that leaves, in the same scale, `low` elements further on
    int64_t ld, low; // low = 0: not split
    uint16_t *turned; // h transposed, for small products (or nullptr), rows of ld_turned
    int64_t ld_turned;
};

__device__ __forceinline__ void put_half(uint16_t *high, uint16_t *low, bool split, const float (&v)[4])
{
    float s[4], back[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = v[i] * pow2(SX);
    const u32x2 h = f16_four(s);
    *reinterpret_cast<u32x2 *>(high) = h;
    if (!split) return;
    f16_values(h, back);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] -= back[i];
    *reinterpret_cast<u32x2 *>(low) = f16_four(s);
}

// The first iterate: U over its norm.
__global__ __launch_bounds__(256) void k_first(source_t s, const double *part, int parts, float eps, iterate_t to, int64_t rows_pad, int64_t cols_pad)
{
    __shared__ double of_wave[4];
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) sum += part[i];
#pragma unroll
    for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = sum;
    __syncthreads();
    const double inverse = 1.0 / (sqrt(of_wave[0] + of_wave[1] + of_wave[2] + of_wave[3]) + eps);
    const int64_t pieces = cols_pad / 8, all = rows_pad * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces, c = (i - r * pieces) * 8;
        const int n = r < s.rows ? (int)(s.cols - c < 8 ? s.cols - c : 8) : 0;
        float u[8] = {};
        if (n > 0) u_at(s, s.m_out, r, c, n, false, u);
        float lo[4], hi[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            lo[k] = k < n ? (float)(u[k] * inverse) : 0.0f;
            hi[k] = k + 4 < n ? (float)(u[k + 4] * inverse) : 0.0f;
        }
        const int64_t at = r * to.ld + c;
        *reinterpret_cast<float4 *>(to.x + at) = make_float4(lo[0], lo[1], lo[2], lo[3]);
        *reinterpret_cast<float4 *>(to.x + at + 4) = make_float4(hi[0], hi[1], hi[2], hi[3]);
        put_half(to.h + at, to.h + to.low + at, to.low != 0, lo);
        put_half(to.h + at + 4, to.h + to.low + at + 4, to.low != 0, hi);
    }
}

// Eight elements of a column of the iterate as part of a row of its transpose.
__device__ __forceinline__ void put_half_turned(const iterate_t &t, int64_t c, int64_t r, const float (&v)[8])
{
    uint16_t *const to = t.turned + c * t.ld_turned + r;
    float lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) lo[i] = v[i], hi[i] = v[i + 4];
    put_half(to, to + t.low, t.low != 0, lo);
    put_half(to + 4, to + 4 + t.low, t.low != 0, hi);
}

// k_first for small products: the transpose as well, 64 x 64 elements a workgroup.
__global__ __launch_bounds__(256) void k_first_turned(source_t s, const double *part, int parts, float eps, iterate_t to)
{
    __shared__ double of_wave[4];
    __shared__ float tile[64][65];
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) sum += part[i];
#pragma unroll
    for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
    if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = sum;
    __syncthreads();
    const double inverse = 1.0 / (sqrt(of_wave[0] + of_wave[1] + of_wave[2] + of_wave[3]) + eps);
    const int64_t r0 = (int64_t)blockIdx.x * 64, c0 = (int64_t)blockIdx.y * 64;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int i = (threadIdx.x >> 3) + 32 * p, j = (threadIdx.x & 7) * 8;
        const int64_t r = r0 + i, c = c0 + j, at = r * to.ld + c;
        const int n = r < s.rows ? (int)(s.cols - c < 8 ? s.cols - c : 8) : 0;
        float u[8] = {};
        if (n > 0) u_at(s, s.m_out, r, c, n, false, u);
        float lo[4], hi[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            tile[i][j + k] = lo[k] = k < n ? (float)(u[k] * inverse) : 0.0f;
            tile[i][j + k + 4] = hi[k] = k + 4 < n ? (float)(u[k + 4] * inverse) : 0.0f;
        }
        *reinterpret_cast<float4 *>(to.x + at) = make_float4(lo[0], lo[1], lo[2], lo[3]);
        *reinterpret_cast<float4 *>(to.x + at + 4) = make_float4(hi[0], hi[1], hi[2], hi[3]);
        put_half(to.h + at, to.h + to.low + at, to.low != 0, lo);
        put_half(to.h + at + 4, to.h + to.low + at + 4, to.low != 0, hi);
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int j = (threadIdx.x >> 3) + 32 * p, i = (threadIdx.x & 7) * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = tile[i + k][j];
        put_half_turned(to, c0 + j, r0 + i, v);
    }
}

// ---- what becomes of the products ---------------------------------------------------------------------------------------------------
// X X^T: its diagonal, and the rest in fp16.
struct gram_t {
    static constexpr bool COUNTED = false;
    static constexpr int AHEAD = 2;
    typedef nothing_t column_t, more_t;
    uint16_t *O;
    float *D;
    int64_t ld;
    __device__ __forceinline__ column_t column(int64_t, int) const { return {}; }
    __device__ __forceinline__ more_t get(const spot_t &, int) const { return {}; }
    __device__ __forceinline__ float4 apply(const spot_t &s, int, float4 v, column_t, more_t) const
    {
        const int64_t r = s.row(), c = s.col();
        float o[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (r == c + i) {
                D[r] = o[i] * pow2(-2 * SX);
                o[i] = 0.0f;
            }
            o[i] *= pow2(SO - 2 * SX);
        }
        *reinterpret_cast<u32x2 *>(s.in(O, ld)) = f16_four(o);
        return make_float4(o[0], o[1], o[2], o[3]);
    }
    __device__ __forceinline__ void put_turned(int64_t c, int64_t r, const float (&v)[8]) const { store_eight(O + c * ld + r, v); }
};

// O O: the polynomial's off-diagonal part in fp16, its diagonal (with a) in fp32.
struct poly_t {
    static constexpr bool COUNTED = false;
    static constexpr int AHEAD = 2;
    const uint16_t *O;
    const float *D;
    uint16_t *P;
    float *diagonal;
    int64_t ld;
    float a, b, c;
    typedef float4 column_t;
    struct more_t {
        u32x2 o;
        float dr;
    };
    __device__ __forceinline__ column_t column(int64_t col, int) const { return *reinterpret_cast<const float4 *>(D + col); }
    __device__ __forceinline__ more_t get(const spot_t &s, int) const { return {*reinterpret_cast<const u32x2 *>(s.in(O, ld)), D[s.row()]}; }
    __device__ __forceinline__ float4 apply(const spot_t &at, int, float4 v, const column_t &d, const more_t &m) const
    {
        const int64_t r = at.row(), col = at.col();
        const float sq[4] = {v.x, v.y, v.z, v.w}, dc[4] = {d.x, d.y, d.z, d.w};
        float o[4], p[4];
        f16_values(m.o, o);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float s = sq[i] * pow2(-2 * SO);
            o[i] *= pow2(-SO);
            p[i] = (b * o[i] + c * ((m.dr + dc[i]) * o[i] + s)) * pow2(SB);
            if (r == col + i) {
                diagonal[r] = a + (b * m.dr + c * (m.dr * m.dr + s));
                p[i] = 0.0f;
            }
        }
        *reinterpret_cast<u32x2 *>(at.in(P, ld)) = f16_four(p);
        return make_float4(p[0], p[1], p[2], p[3]);
    }
    __device__ __forceinline__ void put_turned(int64_t col, int64_t r, const float (&v)[8]) const { store_eight(P + col * ld + r, v); }
};

// In a step whose noise many others multiply, the diagonal of b A + c A^2 takes X as the products take it, in fp16, and a alone the carried one.  X of few directions, X = u v^T say,
// has P X = p u (u^T X) with P = b A + c A^2 for whatever X holds, also for its rounding N: along u.  With P's diagonal times the exact X, - p diag(u^2) N is left, in directions that
// X does not have, and each later step multiplies those by a.  (160 x 200 of one direction: 2.7e-3 of the result's norm off after five steps
// and 6.9e-2 after eight; this way 4e-4 and 1e-3.)
// Where A is mostly diagonal the exact X is what is better, so the last steps have it: iterate() decides.
struct as_rounded_t {
    float a;
    int on;
    __device__ __forceinline__ void put_right(const float (&x)[4], const float (&d)[4], float (&n)[4]) const
    {
        if (!on) return;
        float s[4], back[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = x[i] * pow2(SX);
        f16_values(f16_four(s), back);
#pragma unroll
        for (int i = 0; i < 4; ++i) n[i] += (d[i] - a) * (back[i] * pow2(-SX) - x[i]);
    }
};

// The next iterate's elements from the product's and the carried ones.  BY_ROW: the diagonal goes by rows (A = X X^T), else by columns.
template <bool BY_ROW> struct carried_t;

template <> struct carried_t<true> {
    typedef nothing_t column_t;
    struct more_t {
        float4 x;
        float d;
    };
    const float *x, *diagonal;
    int64_t ld;
    as_rounded_t as;
    __device__ __forceinline__ column_t column(int64_t, int) const { return {}; }
    __device__ __forceinline__ more_t get(const spot_t &s) const { return {*reinterpret_cast<const float4 *>(s.in(x, ld)), diagonal[s.row()]}; }
    __device__ __forceinline__ void next(float4 v, column_t, const more_t &m, float (&n)[4]) const
    {
        const float k = pow2(-SB - SX), x4[4] = {m.x.x, m.x.y, m.x.z, m.x.w}, d[4] = {m.d, m.d, m.d, m.d};
        n[0] = m.d * m.x.x + v.x * k, n[1] = m.d * m.x.y + v.y * k, n[2] = m.d * m.x.z + v.z * k, n[3] = m.d * m.x.w + v.w * k;
        as.put_right(x4, d, n);
    }
};

template <> struct carried_t<false> {
    typedef float4 column_t, more_t;
    const float *x, *diagonal;
    int64_t ld;
    as_rounded_t as;
    __device__ __forceinline__ column_t column(int64_t c, int) const { return *reinterpret_cast<const float4 *>(diagonal + c); }
    __device__ __forceinline__ more_t get(const spot_t &s) const { return *reinterpret_cast<const float4 *>(s.in(x, ld)); }
    __device__ __forceinline__ void next(float4 v, const column_t &d, const more_t &x, float (&n)[4]) const
    {
        const float k = pow2(-SB - SX), x4[4] = {x.x, x.y, x.z, x.w}, d4[4] = {d.x, d.y, d.z, d.w};
        n[0] = d.x * x.x + v.x * k, n[1] = d.y * x.y + v.y * k, n[2] = d.z * x.z + v.z * k, n[3] = d.w * x.w + v.w * k;
        as.put_right(x4, d4, n);
    }
};

template <bool BY_ROW> struct step_t { // the next iterate; x in place
    static constexpr bool COUNTED = false;
    static constexpr int AHEAD = 2;
    typedef typename carried_t<BY_ROW>::column_t column_t;
    typedef typename carried_t<BY_ROW>::more_t more_t;
    carried_t<BY_ROW> from;
    iterate_t to;
    __device__ __forceinline__ column_t column(int64_t c, int have) const { return from.column(c, have); }
    __device__ __forceinline__ more_t get(const spot_t &s, int) const { return from.get(s); }
    __device__ __forceinline__ float4 apply(const spot_t &s, int, float4 v, const column_t &d, const more_t &m) const
    {
        float n[4];
        from.next(v, d, m, n);
        *reinterpret_cast<float4 *>(s.in(to.x, to.ld)) = make_float4(n[0], n[1], n[2], n[3]);
        uint16_t *const h = s.in(to.h, to.ld);
        put_half(h, h + to.low, to.low != 0, n);
        return make_float4(n[0], n[1], n[2], n[3]);
    }
    __device__ __forceinline__ void put_turned(int64_t c, int64_t r, const float (&v)[8]) const { put_half_turned(to, c, r, v); }
};

template <bool BY_ROW> struct result_t { // the last one, as the result
    static constexpr bool COUNTED = false;
    static constexpr int AHEAD = 2;
    typedef typename carried_t<BY_ROW>::column_t column_t;
    typedef typename carried_t<BY_ROW>::more_t more_t;
    carried_t<BY_ROW> from;
    adahop_tensor_t out;
    int64_t rows, cols;
    float scale;
    __device__ __forceinline__ column_t column(int64_t c, int have) const { return from.column(c, have); }
    __device__ __forceinline__ more_t get(const spot_t &s, int) const { return from.get(s); }
    __device__ __forceinline__ float4 apply(const spot_t &at, int, float4 v, const column_t &d, const more_t &m) const
    {
        if (at.row() >= rows || at.col() >= cols) return v;
        float n[4];
        from.next(v, d, m, n);
#pragma unroll
        for (int i = 0; i < 4; ++i) n[i] *= scale;
        put4_at(out, at, (int)(cols - at.col() < 4 ? cols - at.col() : 4), n);
        return v;
    }
};

template <bool BY_ROW> struct update_t { // the last one, as a step of the weight
    static constexpr bool COUNTED = false;
    static constexpr int AHEAD = 1; // a block more does not fit the registers: 28672 x 8192 3.83 ms instead of 3.65
    typedef typename carried_t<BY_ROW>::column_t column_t;
    carried_t<BY_ROW> from;
    adahop_tensor_t w, out, copy; // copy: bf16, or absent
    int64_t rows, cols;
    float keep, rate;
    struct more_t {
        typename carried_t<BY_ROW>::more_t x;
        float4 w;
    };
    __device__ __forceinline__ column_t column(int64_t c, int have) const { return from.column(c, have); }
    __device__ __forceinline__ more_t get(const spot_t &s, int) const
    {
        more_t m;
        m.x = from.get(s);
        m.w = s.row() < rows && s.col() < cols ? get4_at(w, s, (int)(cols - s.col() < 4 ? cols - s.col() : 4)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        return m;
    }
    __device__ __forceinline__ float4 apply(const spot_t &at, int, float4 v, const column_t &d, const more_t &m) const
    {
        if (at.row() >= rows || at.col() >= cols) return v;
        const int have = (int)(cols - at.col() < 4 ? cols - at.col() : 4);
        float n[4];
        from.next(v, d, m.x, n);
        n[0] = keep * m.w.x - rate * n[0], n[1] = keep * m.w.y - rate * n[1], n[2] = keep * m.w.z - rate * n[2], n[3] = keep * m.w.w - rate * n[3];
        put4_at(out, at, have, n);
        if (copy.data) put4_at(copy, at, have, n);
        return v;
    }
};

// ---- host ----------------------------------------------------------------------------------------------------------------------------
struct ns_plan_t {
    bool wide, split, gram_direct, poly_direct, step_direct; // direct: by k_direct16
    bool keeps_turned;                                       // the iterate's transpose is kept for them
    int64_t rows, cols, side, length; // padded: the matrix's, the smaller one and the larger
    int64_t ld, ld_side, ld_turned;   // of the iterate's rows, of the square matrices', of the iterate's transpose's
    plan16_t gram, poly, step;
    int64_t half; // elements from an iterate's high half to its low one
    size_t sums, D, diagonal, O, P, x, h[2], turned[2], part, total;
};

// Rows of a multiple of 8 KB of 16-bit elements are held a line further apart: a slab's pieces of all rows would lie in few of the caches' channels.
int64_t row_pitch(int64_t elements) { return elements % 4096 ? elements : elements + 64; }

ns_plan_t ns_plan(int64_t rows, int64_t cols)
{
    ns_plan_t p;
    p.wide = rows <= cols;
    p.rows = align_up(rows, SLAB), p.cols = align_up(cols, SLAB);
    p.side = p.wide ? p.rows : p.cols, p.length = p.wide ? p.cols : p.rows;
    p.split = (p.wide ? rows : cols) <= SPLIT_SIDE;
    p.ld = row_pitch(p.cols), p.ld_side = row_pitch(p.side), p.ld_turned = row_pitch(p.rows);
    const int64_t long_k = p.length * (p.split ? 3 : 1), side_k = p.side * (p.split ? 2 : 1);
    p.gram = plan16(p.side, p.side, long_k, true, 64, p.split);
    p.poly = plan16(p.side, p.side, p.side, true);
    p.step = plan16(p.rows, p.cols, side_k, false, 64, p.split);
    const plan16_t gram = plan_direct16(p.side, p.side, long_k, true), poly = plan_direct16(p.side, p.side, p.side, true), step = plan_direct16(p.rows, p.cols, side_k, false);
    // k_direct16 wants both operands by rows: the iterate's transpose for the step of a wide matrix, for A of a tall one.  It is the step that writes it, running there itself: a tall
    // matrix has both there or neither.  A of a split wide matrix (one tile of 128, both operands by rows) is always better off there.
    p.poly_direct = poly.time < p.poly.time;
    if (p.wide) {
        p.gram_direct = p.split || gram.time < p.gram.time;
        p.step_direct = step.time < p.step.time;
    } else
        p.gram_direct = p.step_direct = gram.time + step.time < p.gram.time + p.step.time;
    p.keeps_turned = p.step_direct;
    if (p.gram_direct) p.gram = gram;
    if (p.poly_direct) p.poly = poly;
    if (p.step_direct) p.step = step;
    size_t part = p.gram.part_bytes;
    for (const plan16_t *q : {&p.poly, &p.step})
        if (q->part_bytes > part) part = q->part_bytes;
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at = align_up(at + bytes, 256);
        return here;
    };
    const size_t by_rows = (size_t)p.rows * p.ld, by_cols = (size_t)p.cols * p.ld_turned, all = by_rows > by_cols ? by_rows : by_cols, square = (size_t)p.side * p.ld_side;
    p.half = (int64_t)all;
    p.sums = take(PARTS * sizeof(double));
    p.D = take(p.side * sizeof(float));
    p.diagonal = take(p.side * sizeof(float));
    p.O = take(square * 2);
    p.P = take(square * 2);
    p.x = take(all * sizeof(float));
    for (size_t &h : p.h) h = take(all * 2 * (p.split ? 2 : 1));
    for (size_t &h : p.turned) h = take(p.keeps_turned ? all * 2 * (p.split ? 2 : 1) : 0);
    p.part = take(part);
    p.total = at;
    return p;
}

device_once_t g_once;

template <bool SEG> int configure_some()
{
    int rc = ADAHOP_OK;
    if constexpr (!SEG) rc = configure_all16<true, ALONG, ALONG, SEG, true, gram_t>();
    if (rc == ADAHOP_OK) rc = configure_all16<true, DOWN, DOWN, SEG, true, gram_t>();
    if (rc == ADAHOP_OK) rc = configure_all16<true, ALONG, DOWN, SEG, false, step_t<true>>();
    if (rc == ADAHOP_OK) rc = configure_all16<true, ALONG, ALONG, SEG, false, step_t<false>>();
    if (rc == ADAHOP_OK) rc = configure_all16<true, ALONG, DOWN, SEG, false, result_t<true>>();
    if (rc == ADAHOP_OK) rc = configure_all16<true, ALONG, ALONG, SEG, false, result_t<false>>();
    if (rc == ADAHOP_OK) rc = configure_all16<true, ALONG, DOWN, SEG, false, update_t<true>>();
    if (rc == ADAHOP_OK) rc = configure_all16<true, ALONG, ALONG, SEG, false, update_t<false>>();
    if (rc == ADAHOP_OK) rc = configure_direct16<true, SEG, true, true, gram_t>();
    if (rc == ADAHOP_OK) rc = configure_direct16<true, SEG, false, true, step_t<true>>();
    if (rc == ADAHOP_OK) rc = configure_direct16<true, SEG, false, true, step_t<false>>();
    if (rc == ADAHOP_OK) rc = configure_direct16<true, SEG, false, false, result_t<true>>();
    if (rc == ADAHOP_OK) rc = configure_direct16<true, SEG, false, false, result_t<false>>();
    if (rc == ADAHOP_OK) rc = configure_direct16<true, SEG, false, false, update_t<true>>();
    if (rc == ADAHOP_OK) rc = configure_direct16<true, SEG, false, false, update_t<false>>();
    return rc;
}

// The products of one call.
struct ns_call_t {
    ns_plan_t p;
    char *ws;
    hipStream_t st;
    iterate_t at(int which) const
    {
        return {reinterpret_cast<float *>(ws + p.x), reinterpret_cast<uint16_t *>(ws + p.h[which]), p.ld, p.split ? p.half : 0,
                p.keeps_turned ? reinterpret_cast<uint16_t *>(ws + p.turned[which]) : nullptr, p.ld_turned};
    }
    float *D() const { return reinterpret_cast<float *>(ws + p.D); }
    float *diagonal() const { return reinterpret_cast<float *>(ws + p.diagonal); }
    uint16_t *O() const { return reinterpret_cast<uint16_t *>(ws + p.O); }
    uint16_t *P() const { return reinterpret_cast<uint16_t *>(ws + p.P); }

    template <bool SEG> int gram(int which) const
    {
        const iterate_t x = at(which);
        product_t q = {};
        q.A = q.B = {x.h, x.ld, p.side};
        q.K = p.length;
        q.seg = {3, {0, 0, x.low}, {0, x.low, 0}}; // high high + high low + low high
        const gram_t e = {O(), D(), p.ld_side};
        if (p.gram_direct) {
            if (!p.wide) q.A = q.B = {x.turned, x.ld_turned, p.side};
            return launch_direct16<true, SEG, true, true>(p.gram, q, e, ws + p.part, st);
        }
        if constexpr (!SEG)
            if (p.wide) return launch_product16<true, ALONG, ALONG, SEG, true>(p.gram, q, e, ws + p.part, st);
        return launch_product16<true, DOWN, DOWN, SEG, true>(p.gram, q, e, ws + p.part, st);
    }
    int poly(const float (&k)[3]) const
    {
        product_t q = {};
        q.A = q.B = {O(), p.ld_side, p.side};
        q.K = p.side;
        const poly_t e = {O(), D(), P(), diagonal(), p.ld_side, k[0], k[1], k[2]};
        return p.poly_direct ? launch_direct16<true, false, true, true>(p.poly, q, e, ws + p.part, st) : launch_product16<true, ALONG, ALONG, false, true>(p.poly, q, e, ws + p.part, st);
    }
    // P X (wide), X P: with P symmetric, its rows serve as its columns
    template <bool SEG, bool WIDE, bool TURNED, class E> int step(int which, const E &e) const
    {
        const iterate_t x = at(which);
        product_t q = {};
        q.K = p.side;
        if (p.step_direct) {
            const side_t square = {P(), p.ld_side, p.side};
            if (WIDE)
                q.A = square, q.B = {x.turned, x.ld_turned, p.cols}, q.seg = {2, {0, 0, 0}, {0, x.low, 0}};
            else
                q.A = {x.h, x.ld, p.rows}, q.B = square, q.seg = {2, {0, x.low, 0}, {0, 0, 0}};
            return launch_direct16<true, SEG, false, TURNED>(p.step, q, e, ws + p.part, st);
        }
        if constexpr (WIDE) {
            q.A = {P(), p.ld_side, p.rows}, q.B = {x.h, x.ld, p.cols};
            q.seg = {2, {0, 0, 0}, {0, x.low, 0}};
            return launch_product16<true, ALONG, DOWN, SEG, false>(p.step, q, e, ws + p.part, st);
        } else {
            q.A = {x.h, x.ld, p.rows}, q.B = {P(), p.ld_side, p.cols};
            q.seg = {2, {0, x.low, 0}, {0, 0, 0}};
            return launch_product16<true, ALONG, ALONG, SEG, false>(p.step, q, e, ws + p.part, st);
        }
    }
};

template <bool SEG, bool WIDE> int iterate(const ns_call_t &c, const adahop_newton_schulz_t &m, const adahop_tensor_t &out, const adahop_muon_t *u)
{
    const float k[3] = {m.a, m.b, m.c};
    for (int i = 0; i < m.steps; ++i) {
        // As long as later steps multiply what X lacks by more than 4: with the usual coefficients all but the last two.  (All of them: matrices of no preferred directions are 1.4e-3 off after five steps
        // instead of 0.8e-3; none or all but the last three: those of half of the directions 4e-3 instead of 1.5e-3; by a
        // model of the roundings.)
        const bool rounded = !SEG && pow(fabs((double)m.a), m.steps - 1 - i) > 4.0;
        int rc = c.gram<SEG>(i & 1);
        if (rc == ADAHOP_OK) rc = c.poly(k);
        if (rc != ADAHOP_OK) return rc;
        const carried_t<WIDE> from = {c.at(0).x, c.diagonal(), c.p.ld, {m.a, rounded}};
        if (i + 1 < m.steps)
            rc = c.step<SEG, WIDE, true>(i & 1, step_t<WIDE>{from, c.at((i & 1) ^ 1)});
        else if (u)
            rc = c.step<SEG, WIDE, false>(i & 1, update_t<WIDE>{from, u->w, u->w_out, u->w_bf16, u->rows, u->cols, 1.0f - u->rate * u->weight_decay, u->rate * m.scale});
        else
            rc = c.step<SEG, WIDE, false>(i & 1, result_t<WIDE>{from, out, m.rows, m.cols, m.scale});
        if (rc != ADAHOP_OK) return rc;
    }
    return ADAHOP_OK;
}

} // namespace

int configure_newton_schulz()
{
    int dev = 0;
    int rc = check_hip(hipGetDevice(&dev));
    if (rc != ADAHOP_OK || !g_once.need(dev)) return rc;
    rc = configure_some<false>();
    if (rc == ADAHOP_OK) rc = configure_some<true>();
    if (rc == ADAHOP_OK) rc = configure_all16<true, ALONG, ALONG, false, true, poly_t>();
    if (rc == ADAHOP_OK) rc = configure_direct16<true, false, true, true, poly_t>();
    if (rc == ADAHOP_OK) g_once.mark(dev);
    return rc;
}

size_t newton_schulz_workspace_bytes(int64_t rows, int64_t cols) { return ns_plan(rows, cols).total; }

void newton_schulz_plan(int64_t rows, int64_t cols, int product, int *tile, int *alone, int *slices)
{
    const ns_plan_t p = ns_plan(rows, cols);
    const plan16_t &q = product == 0 ? p.gram : product == 1 ? p.poly : p.step;
    *tile = q.edge, *alone = alone16(q), *slices = (int)q.slices;
}

int launch_newton_schulz(const adahop_newton_schulz_t &m, const adahop_tensor_t &g, const adahop_tensor_t &out, const adahop_muon_t *u, void *workspace, hipStream_t st)
{
    int rc = configure_newton_schulz();
    if (rc != ADAHOP_OK) return rc;
    const ns_call_t c = {ns_plan(m.rows, m.cols), static_cast<char *>(workspace), st};
    source_t s = {g, {}, {}, 0.0f, 0, m.rows, m.cols};
    if (u) s.m = u->momentum, s.m_out = u->momentum_out, s.mu = u->mu, s.nesterov = u->nesterov;
    double *const sums = reinterpret_cast<double *>(c.ws + c.p.sums);
    const int64_t pieces = ceil_div(m.rows * ceil_div(m.cols, 8), 256);
    const int parts = (int)(pieces < PARTS ? pieces : PARTS);
    k_squares<<<parts, 256, 0, st>>>(s, sums);
    if ((rc = check_launch()) != ADAHOP_OK) return rc;
    const int64_t blocks = ceil_div(c.p.rows * (c.p.cols / 8), 256);
    if (c.p.keeps_turned)
        k_first_turned<<<dim3((unsigned)(c.p.rows / 64), (unsigned)(c.p.cols / 64)), 256, 0, st>>>(s, sums, parts, m.eps, c.at(0));
    else
        k_first<<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, st>>>(s, sums, parts, m.eps, c.at(0), c.p.rows, c.p.cols);
    if ((rc = check_launch()) != ADAHOP_OK) return rc;
    if (c.p.split) return c.p.wide ? iterate<true, true>(c, m, out, u) : iterate<true, false>(c, m, out, u);
    return c.p.wide ? iterate<false, true>(c, m, out, u) : iterate<false, false>(c, m, out, u);
}

} // namespace adahop

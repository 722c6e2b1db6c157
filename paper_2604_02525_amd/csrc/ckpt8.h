// Device helpers of the training operators: rows of bf16 or fp32 in pieces of 8 elements per lane, and the 8-bit
// checkpoint format (E4M3 elements, one E8M0 scale per 32 consecutive features of a row).
#pragma once
#include "common.h"

namespace adahop {

namespace {

// Rows may begin at any element: accesses of 16 bytes are declared with the alignment of one element, which costs the
// instruction nothing (one global_load_dwordx4 either way).
typedef uint32_t u32x4_e2 __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef uint32_t u32x4_e4 __attribute__((ext_vector_type(4), aligned(4), may_alias));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2), may_alias));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4), may_alias));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

// Eight elements as they lie in memory.
template <bool F32> struct raw8 {
    u32x4 w[F32 ? 2 : 1];
};

template <bool F32> __device__ __forceinline__ raw8<F32> zero8()
{
    raw8<F32> r;
    r.w[0] = 0;
    if constexpr (F32) r.w[1] = 0;
    return r;
}

// The n >= 1 elements at element `at` of `base`; those from n on count as zero.  ODD = false: n is 8, as
// everywhere in rows of whole pieces.
template <bool F32, bool ODD = true> __device__ __forceinline__ raw8<F32> load8(const void *base, int64_t at, int n)
{
    raw8<F32> r;
    if constexpr (F32) {
        const uint32_t *const p = static_cast<const uint32_t *>(base) + at;
        if (!ODD || n >= 8) {
            r.w[0] = *reinterpret_cast<const u32x4_e4 *>(p);
            r.w[1] = *reinterpret_cast<const u32x4_e4 *>(p + 4);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) r.w[i >> 2][i & 3] = i < n ? p[i] : 0;
        }
    } else {
        const uint16_t *const p = static_cast<const uint16_t *>(base) + at;
        if (!ODD || n >= 8) {
            r.w[0] = *reinterpret_cast<const u32x4_e2 *>(p);
        } else {
            uint32_t e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = i < n ? p[i] : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) r.w[0][i] = e[2 * i] | e[2 * i + 1] << 16;
        }
    }
    return r;
}

template <bool F32> __device__ __forceinline__ void widen8(const raw8<F32> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (F32)
            v[i] = __uint_as_float(r.w[i >> 2][i & 3]);
        else
            v[i] = i & 1 ? bf16_hi(r.w[0][i >> 1]) : bf16_lo(r.w[0][i >> 1]);
    }
}

// How many elements to load of a row's last piece, of which n exist: where another row of the tensor follows, all eight can be read at once and
// those from n on be taken out later.  Element by element the loads of that piece keep the whole workgroup waiting: 8192 x 4091 with both
// checkpoints forward 109 us instead of 91, backward 123 instead of 88.
__device__ __forceinline__ int to_load(int n, bool row_follows, int64_t cols) { return row_follows && cols >= 8 && n > 0 ? 8 : n; }

// Values from the n-th of eight on are zero, whatever they were.
__device__ __forceinline__ void zero_from(int n, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] : 0.0f;
}

// Keeps eight elements as they lie in memory: what has been made of them so far is not kept in registers for later.
template <bool F32> __device__ __forceinline__ void keep_raw(raw8<F32> &r)
{
    asm volatile("" : "+v"(r.w[0]));
    if constexpr (F32) asm volatile("" : "+v"(r.w[1]));
}

// Eight elements of a tensor whose type is known at run time only: for what is read once, or seldom.
template <bool ODD = true> __device__ __forceinline__ void load8_any(const adahop_tensor_t &t, int64_t at, int n, float (&v)[8])
{
    if (t.f32) {
        widen8<true>(load8<true, ODD>(t.data, at, n), v);
    } else {
        widen8<false>(load8<false, ODD>(t.data, at, n), v);
    }
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) // round to nearest even
{
    const v2bf p = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, p);
}

// The first n >= 1 of eight values, rounded once where the tensor is bf16.
template <bool F32, bool ODD = true> __device__ __forceinline__ void store8(void *base, int64_t at, int n, const float (&v)[8])
{
    if constexpr (F32) {
        float *const p = static_cast<float *>(base) + at;
        if (!ODD || n >= 8) {
            u32x4 lo, hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo[i] = __float_as_uint(v[i]);
                hi[i] = __float_as_uint(v[i + 4]);
            }
            *reinterpret_cast<u32x4_e4 *>(p) = lo;
            *reinterpret_cast<u32x4_e4 *>(p + 4) = hi;
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < n) p[i] = v[i];
        }
    } else {
        uint16_t *const p = static_cast<uint16_t *>(base) + at;
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
        if (!ODD || n >= 8) {
            *reinterpret_cast<u32x4_e2 *>(p) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < n) p[i] = (uint16_t)(w[i >> 1] >> 16 * (i & 1));
        }
    }
}

template <bool ODD = true> __device__ __forceinline__ void store8_any(const adahop_tensor_t &t, int64_t at, int n, const float (&v)[8])
{
    if (t.f32)
        store8<true, ODD>(t.data, at, n, v);
    else
        store8<false, ODD>(t.data, at, n, v);
}

template <int CTRL> __device__ __forceinline__ uint32_t max_with(uint32_t m)
{
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, CTRL, 0xf, 0xf, true);
    return m > o ? m : o;
}

// ---- the 8-bit format -------------------------------------------------------------------------------------------------
// Block of 32 features with largest finite magnitude amax: scale = 2^(floor(log2 amax) - 8), the power of two that puts amax
// into E4M3's last binade [256, 512); elements to nearest even, those above 448 saturate.  E4M3 keeps three bits behind the leading one over
// 2^-6 .. 448, so an outlier of 2^8 times its neighbours costs them nothing, which eight-bit integers of one scale would not
// allow.  Infinities and NaN become NaN (E4M3 has no infinity) and do not take part in the scale.
//
// Four neighbouring lanes hold a block.  All lanes of a group of four take part, those without elements with zeros.
struct packed8 {
    u32x2 codes;
    uint8_t scale;
};

__device__ __forceinline__ packed8 pack8(const float (&v)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
        m = m > a ? m : a;
    }
    m = max_with<0xB1 /* quad_perm:[1,0,3,2] */>(m);
    m = max_with<0x4E /* quad_perm:[2,3,0,1] */>(m);
    const bool odd = __builtin_amdgcn_ballot_w64(m >= 0x7f800000u) != 0; // of the wave: hardly ever
    if (odd) {
        m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
            m = a < 0x7f800000u && a > m ? a : m;
        }
        m = max_with<0xB1>(m);
        m = max_with<0x4E>(m);
    }
    const uint32_t e = m >> 23, scale = (e > 8 ? e : 8) - 8;          // zeros and what lies below 2^-118: 2^-127
    const float inverse = __uint_as_float((254 - scale) << 23);
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __builtin_amdgcn_fmed3f(v[i] * inverse, -448.0f, 448.0f);
    if (odd) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((__float_as_uint(v[i]) & 0x7fffffffu) >= 0x7f800000u) q[i] = __uint_as_float(0x7fc00000u);
    }
    packed8 p;
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
    p.codes.x = (uint32_t)lo;
    p.codes.y = (uint32_t)hi;
    p.scale = (uint8_t)scale;
    return p;
}

// Of the piece of n elements that begins at column c (a multiple of 8) of a row.
template <bool ODD = true> __device__ __forceinline__ void store_packed8(const adahop_ckpt8_t &k, int64_t row, int c, int n, const packed8 &p)
{
    uint8_t *const at = k.codes + row * k.ld_codes + c;
    if (!ODD || n >= 8) {
        __builtin_nontemporal_store(p.codes, reinterpret_cast<u32x2 *>(at)); // read by the backward pass, not by what follows: out of the caches' way
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) at[i] = (uint8_t)(p.codes[i >> 2] >> 8 * (i & 3));
    }
    if ((c & 31) == 0) k.scales[row * k.ld_scales + (c >> 5)] = p.scale;
}

template <bool ODD = true> __device__ __forceinline__ packed8 load_packed8(const adahop_ckpt8_t &k, int64_t row, int c, int n)
{
    packed8 p;
    const uint8_t *const at = k.codes + row * k.ld_codes + c;
    if (!ODD || n >= 8) {
        p.codes = *reinterpret_cast<const u32x2 *>(at);
    } else {
        p.codes = 0;
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) p.codes[i >> 2] |= (uint32_t)at[i] << 8 * (i & 3);
    }
    p.scale = k.scales[row * k.ld_scales + (c >> 5)];
    return p;
}

// 2^(s - 127); 255 is NaN (E8M0 has no infinity).  The same mantissa bit makes 0 2^-127 and 255 NaN.
__device__ __forceinline__ float scale_of(uint8_t s) { return __uint_as_float((uint32_t)s << 23 | (((s + 1u) & 255u) < 2 ? 0x00400000u : 0u)); }

__device__ __forceinline__ void unpack8(const packed8 &p, float (&v)[8])
{
    const float s = scale_of(p.scale);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8((int)p.codes[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)p.codes[i], true);
        v[4 * i] = a.x * s;
        v[4 * i + 1] = a.y * s;
        v[4 * i + 2] = b.x * s;
        v[4 * i + 3] = b.y * s;
    }
}

__device__ __forceinline__ void keep_raw(packed8 &p) { asm volatile("" : "+v"(p.codes)); }

// ---- rows of any width, without regard to where they end ----------------------------------------------------------------
// The blocks of 32 of all rows are numbered through: block b lies in row b / per_row.  Division by multiplication, exact for
// b < 2^31: with 2^(l - 1) < per_row <= 2^l and mul = ceil(2^(31 + l) / per_row), 2 b mul / 2^(32 + l) exceeds b / per_row by less than 1 / per_row.
// Workgroups of PIECES lanes, each with eight elements, lie in rows of `across`: a launch takes fewer than 2^32 lanes along one dimension.
constexpr int PIECES = 256;

struct blocks_t {
    uint32_t total, per_row, mul, across;
    int shift;
};

__device__ __forceinline__ void block_at(const blocks_t &g, uint32_t b, uint32_t *row, uint32_t *in_row)
{
    *row = __umulhi(2 * b, g.mul) >> g.shift;
    *in_row = b - *row * g.per_row;
}

} // namespace

inline blocks_t blocks_of(int64_t rows, int64_t cols)
{
    blocks_t g;
    g.per_row = (uint32_t)ceil_div(cols, 32);
    g.total = (uint32_t)(rows * g.per_row);
    g.shift = 0;
    while (((uint32_t)1 << g.shift) < g.per_row) ++g.shift;
    g.mul = (uint32_t)((((uint64_t)1 << (31 + g.shift)) + g.per_row - 1) / g.per_row);
    const int64_t groups = ceil_div((int64_t)g.total * 4, PIECES);
    g.across = (uint32_t)ceil_div(groups, ceil_div(groups, (int64_t)1 << 23));
    return g;
}

} // namespace adahop

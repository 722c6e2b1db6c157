// Device helpers of the products whose 16-bit operands go to LDS by bounded copies, with tiles of 16 x 16 x 32 matrix instructions: the copies, the transposing
// read, and a result's elements in fours.
#pragma once
#include <type_traits>

#include "ckpt8.h"
#include "gemm_mx_common.h"

namespace adahop {

namespace {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));

constexpr int STAGE = 32; // of the contraction per stage: one matrix instruction's

// What a workgroup reads: `bytes` from `base` on, below 2^31; beyond that zeros.
__device__ __forceinline__ rsrc_t resource(const void *base, uint32_t bytes)
{
    const uint8_t *const p = uniform_ptr(static_cast<const uint8_t *>(base));
    rsrc_t r;
    r.x = (uint32_t)(uint64_t)p;
    r.y = (uint32_t)((uint64_t)p >> 32);
    r.z = __builtin_amdgcn_readfirstlane(bytes);
    r.w = 0x00027000u;
    return r;
}

// Lane i's 16 bytes at voff of the resource land at lds + AT + 16 i; zeros where they lie beyond its end.  (dma16 of gemm_mx_common.h with
// bounds.)  lds: wave-uniform.
template <uint32_t AT> __device__ __forceinline__ void dma16_bounded(rsrc_t r, uint32_t voff, uint32_t lds)
{
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                 :
                 : "v"(voff), "s"(r), "s"(lds), "n"(AT)
                 : "memory", "m0", "scc");
}

template <int N> __device__ __forceinline__ void wait_for_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); } // all but the last N

__device__ __forceinline__ u32x2 transposed(uint32_t lds_addr)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)lds_addr));
}

__device__ __forceinline__ float element(const adahop_tensor_t &t, int64_t at)
{
    return t.f32 ? static_cast<const float *>(t.data)[at] : bf16_one(static_cast<const uint16_t *>(t.data)[at]);
}

// f(i) for i = FROM .. TO - 1, i known at compile time.
template <int FROM, int TO, class F> __device__ __forceinline__ void static_for(F &&f)
{
    if constexpr (FROM < TO) {
        f(std::integral_constant<int, FROM>{});
        static_for<FROM + 1, TO>(f);
    }
}

// add[r, c .. c + have), zeros where there is none
__device__ __forceinline__ float4 get4(const adahop_tensor_t &add, int64_t r, int64_t c, int have)
{
    float o[4] = {};
    if (add.data) {
        const int64_t at = r * add.ld + c;
        if (have == 4 && add.f32) {
            const u32x4 a = *reinterpret_cast<const u32x4_e4 *>(static_cast<const uint32_t *>(add.data) + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(a[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < have) o[i] = element(add, at + i);
        }
    }
    return make_float4(o[0], o[1], o[2], o[3]);
}

// C[r, c .. c + have) = v times scale, plus more.
__device__ __forceinline__ void put4(const adahop_tensor_t &to, int64_t r, int64_t c, int have, const float (&scale)[4], float4 v, float4 more)
{
    const float o[4] = {v.x * scale[0] + more.x, v.y * scale[1] + more.y, v.z * scale[2] + more.z, v.w * scale[3] + more.w};
    const int64_t at = r * to.ld + c;
    if (to.f32) {
        uint32_t *const p = static_cast<uint32_t *>(to.data) + at;
        if (have == 4) {
            const u32x4 w = {__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3])};
            *reinterpret_cast<u32x4_e4 *>(p) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < have) p[i] = __float_as_uint(o[i]);
        }
    } else {
        uint16_t *const p = static_cast<uint16_t *>(to.data) + at;
        const u32x2 w = {bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3])};
        if (have == 4) {
            typedef uint32_t u32x2_e2 __attribute__((ext_vector_type(2), aligned(2), may_alias));
            *reinterpret_cast<u32x2_e2 *>(p) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < have) p[i] = (uint16_t)(w[i >> 1] >> 16 * (i & 1));
        }
    }
}

} // namespace

} // namespace adahop

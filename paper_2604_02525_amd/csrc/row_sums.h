// Sums over the waves of a workgroup that hold one row of a matrix: every thread of them gets them.
#pragma once
#include "common.h"

namespace adahop {

namespace {

constexpr int ROW_THREADS = 1024; // at most

template <int CTRL> __device__ __forceinline__ float plus_dpp(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

__device__ __forceinline__ float sum16(float v) // over the 16 lanes of a row of lanes, in each of them
{
    v = plus_dpp<0xB1 /* quad_perm:[1,0,3,2] */>(v);
    v = plus_dpp<0x4E /* quad_perm:[2,3,0,1] */>(v);
    v = plus_dpp<0x141 /* row_half_mirror */>(v);
    return plus_dpp<0x140 /* row_mirror */>(v);
}

__device__ __forceinline__ float sum64(float v)
{
    typedef unsigned int v2u __attribute__((ext_vector_type(2)));
    v = sum16(v);
    v2u r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false); // the even and the odd rows of 16 lanes
    v = __uint_as_float(r.x) + __uint_as_float(r.y);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// The sums of N values over `waves` waves from `first` on, in one order whatever the timing; all waves of the workgroup take part, each for its row.  Two buffers in turn: a wave that writes into
// one has passed the barrier of the sums in the other, which no wave reaches before it has read these ones' predecessors.
template <int N> struct row_sums_t {
    float part[2][N][ROW_THREADS / 64];
};

template <int N> __device__ __forceinline__ void row_sums(row_sums_t<N> &lds, int &turn, int waves, float (&v)[N], int first = 0)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = sum64(v[i]);
    if (waves == 1) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    turn ^= 1;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) lds.part[turn][i][w] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = sum16((lane & 15) < waves ? lds.part[turn][i][first + (lane & 15)] : 0.0f);
}

} // namespace

} // namespace adahop

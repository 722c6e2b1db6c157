// Weight gradient of a linear layer from the 8-bit checkpoint of its input (paper Eq. 3 with X kept in 8 bits):
//
//     C[n, d] = w[d] sum_t G[t, n] X8[t, d] (+ add[n, d])
//
// on the BF16 matrix cores: an E4M3 element times its power of two is a bf16 number, so nothing is rounded on the way there.
#include "ckpt8.h"
#include "gemm_mx_common.h"

namespace adahop {

namespace {

typedef short v4s __attribute__((ext_vector_type(4)));

constexpr int STEP = 32, TILE = 64; // tokens per stage, rows and columns of C per workgroup

struct wgrad_t {
    adahop_tensor_t G, col_scale, add, C;
    adahop_ckpt8_t x;
    int64_t T, N, D;
};

__device__ __forceinline__ uint4 fragment(const uint16_t *lds, int k0, int c0) // 16 tokens x 32 columns, transposed
{
    const int lane = threadIdx.x & 63, s = lane & 15, t = k0 + 8 * (lane >> 5) + (s >> 2), c = c0 + 16 * ((lane >> 4) & 1) + 4 * (s & 3);
    typedef __attribute__((address_space(3))) v4s *lds_t;
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(lds + t * TILE + c));
    const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)(lds + (t + 4) * TILE + c));
    const u32x2 x = __builtin_bit_cast(u32x2, a), y = __builtin_bit_cast(u32x2, b);
    return make_uint4(x.x, x.y, y.x, y.y);
}

__global__ __launch_bounds__(256) void k_wgrad8(wgrad_t q)
{
    __shared__ __attribute__((aligned(16))) uint16_t g[STEP * TILE], x[STEP * TILE];
    const int64_t n0 = (int64_t)blockIdx.y * TILE, d0 = (int64_t)blockIdx.x * TILE;
    const int tid = threadIdx.x, t = tid >> 3, c = (tid & 7) * 8, w = tid >> 6, wn = (w >> 1) * 32, wd = (w & 1) * 32;
    const int gn = (int)(q.N - n0 - c < 8 ? q.N - n0 - c : 8), xn = (int)(q.D - d0 - c < 8 ? q.D - d0 - c : 8);
    v16f acc = {};
    for (int64_t t0 = 0; t0 < q.T; t0 += STEP) {
        raw8<false> a = zero8<false>();
        float v[8] = {};
        if (t0 + t < q.T) {
            if (gn > 0) a = load8<false>(q.G.data, (t0 + t) * q.G.ld + n0 + c, gn);
            if (xn > 0) unpack8(load_packed8(q.x, t0 + t, (int)d0 + c, xn), v);
        }
        __syncthreads();
        *reinterpret_cast<u32x4 *>(g + t * TILE + c) = a.w[0];
        const u32x4 b = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
        *reinterpret_cast<u32x4 *>(x + t * TILE + c) = b;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < STEP; k += 16) acc = mfma_bf16(fragment(g, k, wn), fragment(x, k, wd), acc);
    }
    const int lane = tid & 63;
    const int64_t d = d0 + wd + (lane & 31);
    if (d >= q.D) return;
    const float scale = !q.col_scale.data ? 1.0f : q.col_scale.f32 ? static_cast<const float *>(q.col_scale.data)[d] : bf16_one(static_cast<const uint16_t *>(q.col_scale.data)[d]);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t n = n0 + wn + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
        if (n >= q.N) continue;
        float v = acc[i] * scale;
        if (q.add.data) v += q.add.f32 ? static_cast<const float *>(q.add.data)[n * q.add.ld + d] : bf16_one(static_cast<const uint16_t *>(q.add.data)[n * q.add.ld + d]);
        if (q.C.f32)
            static_cast<float *>(q.C.data)[n * q.C.ld + d] = v;
        else
            static_cast<uint16_t *>(q.C.data)[n * q.C.ld + d] = (uint16_t)bf16_pair(v, 0.0f);
    }
}

} // namespace

size_t wgrad8_workspace_bytes(int64_t, int64_t, int64_t) { return 0; }

int launch_wgrad8(int64_t T, int64_t N, int64_t D, const adahop_tensor_t &G, const adahop_ckpt8_t &x, const adahop_tensor_t &col_scale,
                  const adahop_tensor_t &add, const adahop_tensor_t &C, void *, hipStream_t st)
{
    const wgrad_t q = {G, col_scale, add, C, x, T, N, D};
    k_wgrad8<<<dim3((unsigned)ceil_div(D, TILE), (unsigned)ceil_div(N, TILE)), 256, 0, st>>>(q);
    return check_launch();
}

} // namespace adahop

// Weight gradient of a linear layer from the 8-bit checkpoint of its input (paper Eq. 3 with X kept in 8 bits):
//
//     C[n, d] = w[d] sum_t G[t, n] X8[t, d] (+ add[n, d])
//
// on the BF16 matrix cores: an E4M3 element times its power of two is a bf16 number, so nothing is rounded on the way there.
// Bound by the matrix cores but for a few tokens, where writing C is.
//
// Both operands have the contraction (tokens) along their rows, the matrix cores want it within a lane: the transposing read of LDS
// (ds_read_b64_tr_b16) turns them, four tokens of a column per lane and read.  So LDS holds both tiles as rows of bf16 columns:
//   G    goes there as it is, by copies that pass no register (16 bytes per lane);
//   X8   goes through registers, where 16 codes of one scale become 32 bytes: half the bytes from memory, and one
//        conversion per workgroup instead of one per wave that reads the tile.
// Rows past the last token read as zero (the bounds of a buffer resource), in both operands: infinities and NaN meet no padding.  Columns past the
// operands' hold whatever is there; they end in elements of C that are not stored.
//
// LDS layout: token t's row at t * row bytes, its pieces of 64 bytes exchanged by t's low two bits: the four rows that a transposing
// read of half a wave touches lie in four different quarters of the banks.
#include "ckpt8.h"
#include "gemm_mx_common.h"

namespace adahop {

namespace {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));

constexpr int STAGE = 64, STEPS = STAGE / 16; // tokens per stage; matrix-core steps in it

struct wgrad_t {
    adahop_tensor_t G, col_scale, add, C;
    adahop_ckpt8_t x;
    int64_t T, N, D;
    float *part;        // [slices][N][D], or nullptr: one slice, finished by the kernel itself
    int64_t slice;      // tokens per slice, whole stages
    uint32_t nt, dt;    // tiles along N and D
};

// What a workgroup reads: `bytes` from `base` on; beyond that zeros.
__device__ __forceinline__ rsrc_t resource(const uint8_t *base, int64_t bytes)
{
    base = uniform_ptr(base);
    const int64_t most = bytes < 0 ? 0 : bytes > 0xfffffffc ? 0xfffffffc : bytes;
    rsrc_t r;
    r.x = (uint32_t)(uint64_t)base;
    r.y = (uint32_t)((uint64_t)base >> 32);
    r.z = __builtin_amdgcn_readfirstlane((uint32_t)most);
    r.w = 0x00027000u;
    return r;
}

// Lane i's 16 bytes at voff of the resource land at lds_addr + 16 i; zeros where they lie beyond its end.  (dma16 of gemm_mx_common.h
// with bounds.)
__device__ __forceinline__ void dma16_bounded(rsrc_t r, uint32_t voff, uint32_t lds_addr)
{
    lds_addr = __builtin_amdgcn_readfirstlane(lds_addr);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                 :
                 : "v"(voff), "s"(r), "s"(lds_addr)
                 : "memory", "m0");
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t typed(rsrc_t r)
{
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>((uint64_t)r.y << 32 | r.x), 0, (int)r.z, (int)r.w);
}

__device__ __forceinline__ u32x2 transposed(uint32_t lds_addr)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)lds_addr));
}

__device__ __forceinline__ float element(const adahop_tensor_t &t, int64_t at)
{
    return t.f32 ? static_cast<const float *>(t.data)[at] : bf16_one(static_cast<const uint16_t *>(t.data)[at]);
}

// Tiles of 64 MT x 64 NT of C by four waves of 32 MT x 32 NT.  Two buffers of a stage each: while a stage is multiplied, the next one's G is
// copied and its X8 is loaded (step 0), converted and written (step 2); one barrier per stage, before step 3, in which the first operands of the
// next stage are read.  The operands of a step are read during the step before it.
template <int MT, int NT> struct tile_t {
    static constexpr int TM = 64 * MT, TN = 64 * NT, RA = 2 * TM, RB = 2 * TN;      // columns; bytes of a row in LDS
    static constexpr uint32_t A = STAGE * RA, B = STAGE * RB, LDS = 2 * (A + B);    // bytes of a buffer; of all four
    static constexpr int COPIES = STAGE * RA / 1024 / 4;                            // of G per wave and stage
    static constexpr int PIECES = STAGE * TN / 16 / 256;                            // of 16 codes per lane and stage
    static constexpr int ROWS_PER_COPY = 1024 / RA, ROWS_PER_PIECE = 256 / (TN / 16);
};

template <int MT, int NT> __global__ __launch_bounds__(256) void k_wgrad8(wgrad_t q)
{
    typedef tile_t<MT, NT> K;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wn = w >> 1, wd = w & 1;
    const uint32_t lds = lds_address(smem);

    // Workgroups go round the eight XCDs; each takes a run of tiles, which it walks in columns of four tiles: what runs on it at a time
    // shares four tiles of G's columns and eight of X's (half as many bytes each).
    const uint32_t tiles = q.nt * q.dt, id = blockIdx.x, per = tiles / 8, rest = tiles % 8, xcd = id % 8;
    const uint32_t t = xcd * per + (xcd < rest ? xcd : rest) + id / 8, group = t / (4 * q.dt), in = t - group * 4 * q.dt;
    const uint32_t high = q.nt - 4 * group < 4 ? q.nt - 4 * group : 4;
    const int64_t n0 = (int64_t)(4 * group + in % high) * K::TM, d0 = (int64_t)(in / high) * K::TN;
    const int64_t begin = (int64_t)blockIdx.y * q.slice, end = begin + q.slice < q.T ? begin + q.slice : q.T;

    // Where this wave's and this lane's parts of a stage lie.
    const uint32_t ld = (uint32_t)(q.G.ld * 2), ldc = (uint32_t)q.x.ld_codes, lds_s = (uint32_t)q.x.ld_scales;
    const int row = w * K::COPIES * K::ROWS_PER_COPY + lane / (K::RA / 16), chunk = lane % (K::RA / 16);
    uint32_t voff[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) // copies of even and odd number
        voff[i] = (uint32_t)row * ld + (((chunk >> 2) ^ ((row + i * K::ROWS_PER_COPY) & 3)) * 64 + (chunk & 3) * 16);
    const int prow = tid / (K::TN / 16), pc = tid % (K::TN / 16);
    const uint8_t *gp = reinterpret_cast<const uint8_t *>(q.G.data) + begin * q.G.ld * 2 + n0 * 2;
    const uint8_t *xp = q.x.codes + begin * q.x.ld_codes + d0, *sp = q.x.scales + begin * q.x.ld_scales + (d0 >> 5);
    int64_t left = end - begin; // tokens from the stage at hand on
    // bytes of a row of the tile that exist, in whole words
    const int64_t ge = ((q.N - n0) * 2 + 3) & ~3LL, xe = (q.D - d0 + 3) & ~3LL, se = (q.D - d0 + 31) >> 5;

    uint32_t copy_to = lds + w * K::COPIES * 1024;
    uint32_t put = lds + 2 * K::A + prow * K::RB + (((pc >> 1) ^ (prow & 3)) * 64 + (pc & 1) * 32);
    const int s16 = lane & 15, h = lane >> 5;
    uint32_t va[MT], vb[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) va[m] = lds + (8 * h + (s16 >> 2)) * K::RA + (((wn * MT + m) ^ (s16 >> 2)) * 64) + 32 * ((lane >> 4) & 1) + 8 * (s16 & 3);
#pragma unroll
    for (int n = 0; n < NT; ++n) vb[n] = lds + 2 * K::A + (8 * h + (s16 >> 2)) * K::RB + (((wd * NT + n) ^ (s16 >> 2)) * 64) + 32 * ((lane >> 4) & 1) + 8 * (s16 & 3);

    u32x4 codes[K::PIECES];
    uint32_t scales[K::PIECES];
    rsrc_t rg, rx, rs;
    const auto aim = [&] { // at the stage that begins at gp, xp, sp
        rg = resource(gp, left > 0 ? (left - 1) * (int64_t)ld + ge : 0);
        rx = resource(xp, left > 0 ? (left - 1) * (int64_t)ldc + xe : 0);
        rs = resource(sp, left > 0 ? (left - 1) * (int64_t)lds_s + se : 0);
    };
    const auto copy = [&](int i) { dma16_bounded(rg, voff[i & 1] + i * K::ROWS_PER_COPY * ld, copy_to + i * 1024); };
    const auto fetch = [&](int j) {
        const uint32_t r = prow + j * K::ROWS_PER_PIECE;
        codes[j] = __builtin_amdgcn_raw_buffer_load_b128(typed(rx), r * ldc + pc * 16, 0, 0);
        scales[j] = __builtin_amdgcn_raw_buffer_load_b8(typed(rs), r * lds_s + (pc >> 1), 0, 0);
    };
    const auto convert = [&](int j, int half) { // eight codes: 16 bytes of LDS
        const float scale = __uint_as_float(scales[j] << 23);
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t four = codes[j][2 * half + i];
            v[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, false));
            v[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, true));
        }
        *(__attribute__((address_space(3))) u32x4 *)(put + j * K::ROWS_PER_PIECE * K::RB + half * 16) = v;
    };
    const auto next = [&] {
        gp += (int64_t)STAGE * ld;
        xp += (int64_t)STAGE * ldc;
        sp += (int64_t)STAGE * lds_s;
        left -= STAGE;
    };
    const auto other_buffer = [&] { // of what is written; what is read follows a step later
        copy_to = lds + ((copy_to - lds) ^ K::A);
        put = lds + 2 * K::A + ((put - lds - 2 * K::A) ^ K::B);
    };

    v16f acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = {};
    u32x2 fa[2][MT][2], fb[2][NT][2];
    // Read number i of a step's operands, in the order in which they are used: G's first tile, all of X's, G's others.
    const auto read = [&](int set, int step, int i) {
        const int tile = i >> 1, part = i & 1;
        if (tile == 0)
            fa[set][0][part] = transposed(va[0] + (16 * step + 4 * part) * K::RA);
        else if (tile <= NT)
            fb[set][tile - 1][part] = transposed(vb[tile - 1] + (16 * step + 4 * part) * K::RB);
        else
            fa[set][tile - NT][part] = transposed(va[tile - NT] + (16 * step + 4 * part) * K::RA);
    };
    constexpr int READS = 2 * (MT + NT), SLOTS = MT * NT;

    if (left > 0) {
        aim();
#pragma unroll
        for (int i = 0; i < K::COPIES; ++i) copy(i);
#pragma unroll
        for (int j = 0; j < K::PIECES; ++j) fetch(j);
#pragma unroll
        for (int j = 0; j < K::PIECES; ++j) {
            convert(j, 0);
            convert(j, 1);
        }
        other_buffer();
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
        for (int i = 0; i < READS; ++i) read(0, 0, i);
    }
    while (left > 0) {
        next();
        aim();
#pragma unroll
        for (int step = 0; step < STEPS; ++step) {
            if (step == STEPS - 1) {
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
                other_buffer();
#pragma unroll
                for (int m = 0; m < MT; ++m) va[m] = lds + ((va[m] - lds) ^ K::A);
#pragma unroll
                for (int n = 0; n < NT; ++n) vb[n] = lds + 2 * K::A + ((vb[n] - lds - 2 * K::A) ^ K::B);
            }
            ADAHOP_PIN();
#pragma unroll
            for (int slot = 0; slot < SLOTS; ++slot) {
                const int m = slot / NT, n = slot % NT, set = step & 1;
                const auto whole = [](const u32x2 (&f)[2]) { return make_uint4(f[0].x, f[0].y, f[1].x, f[1].y); };
                acc[m][n] = mfma_bf16(whole(fa[set][m]), whole(fb[set][n]), acc[m][n]);
#pragma unroll
                for (int i = slot * READS / SLOTS; i < (slot + 1) * READS / SLOTS; ++i) read(set ^ 1, (step + 1) % STEPS, i);
                if (step == 0) {
#pragma unroll
                    for (int i = slot * K::COPIES / SLOTS; i < (slot + 1) * K::COPIES / SLOTS; ++i) copy(i);
#pragma unroll
                    for (int j = slot * K::PIECES / SLOTS; j < (slot + 1) * K::PIECES / SLOTS; ++j) fetch(j);
                }
                if (step == 2) {
#pragma unroll
                    for (int i = slot * 2 * K::PIECES / SLOTS; i < (slot + 1) * 2 * K::PIECES / SLOTS; ++i) convert(i >> 1, i & 1);
                }
                ADAHOP_PIN();
            }
        }
    }

    // lane: column lane % 32 of each tile of 32 x 32, rows 8 (i / 4) + 4 h + i % 4
    const int64_t nb = n0 + wn * MT * 32 + 4 * h, db = d0 + wd * NT * 32 + (lane & 31);
    if (q.part) {
        float *const p = q.part + (int64_t)blockIdx.y * q.N * q.D;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int64_t r = nb + 32 * m + 8 * (i >> 2) + (i & 3), c = db + 32 * n;
                    if (r < q.N && c < q.D) p[r * q.D + c] = acc[m][n][i];
                }
        return;
    }
    float scale[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) scale[n] = q.col_scale.data && db + 32 * n < q.D ? element(q.col_scale, db + 32 * n) : 1.0f;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int64_t r = nb + 32 * m + 8 * (i >> 2) + (i & 3), c = db + 32 * n;
                if (r >= q.N || c >= q.D) continue;
                float v = acc[m][n][i] * scale[n];
                if (q.add.data) v += element(q.add, r * q.add.ld + c);
                if (q.C.f32)
                    static_cast<float *>(q.C.data)[r * q.C.ld + c] = v;
                else
                    static_cast<uint16_t *>(q.C.data)[r * q.C.ld + c] = (uint16_t)bf16_pair(v, 0.0f);
            }
}

// The sums of the slices, in their order, and what the kernel above does with a single one's.
__global__ __launch_bounds__(256) void k_wgrad8_join(wgrad_t q, int slices)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x, r = blockIdx.y + (int64_t)blockIdx.z * 65535;
    if (c >= q.D || r >= q.N) return;
    float v = 0.0f;
    for (int s = 0; s < slices; ++s) v += q.part[((int64_t)s * q.N + r) * q.D + c];
    if (q.col_scale.data) v *= element(q.col_scale, c);
    if (q.add.data) v += element(q.add, r * q.add.ld + c);
    if (q.C.f32)
        static_cast<float *>(q.C.data)[r * q.C.ld + c] = v;
    else
        static_cast<uint16_t *>(q.C.data)[r * q.C.ld + c] = (uint16_t)bf16_pair(v, 0.0f);
}

struct plan_t {
    bool large;     // tiles of 256 x 256, else 128 x 128
    int slices;
    int64_t slice;
};

plan_t plan_of(int64_t T, int64_t N, int64_t D)
{
    const int64_t large = ceil_div(N, 256) * ceil_div(D, 256), small = ceil_div(N, 128) * ceil_div(D, 128), stages = ceil_div(T, STAGE);
    plan_t p;
    p.large = large >= 256;
    const int64_t tiles = p.large ? large : small, fit = 512 / tiles;
    int64_t slices = p.large || fit < 2 ? 1 : fit;
    if (slices > stages / 8) slices = stages / 8;
    if (slices < 1) slices = 1;
    p.slice = ceil_div(stages, slices) * STAGE;
    p.slices = T > 0 ? (int)ceil_div(T, p.slice) : 1;
    return p;
}

device_once_t g_once;

} // namespace

int configure_wgrad8()
{
    int dev = 0;
    int rc = check_hip(hipGetDevice(&dev));
    if (rc != ADAHOP_OK || !g_once.need(dev)) return rc;
    rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void *>(&k_wgrad8<4, 4>), hipFuncAttributeMaxDynamicSharedMemorySize, tile_t<4, 4>::LDS));
    if (rc == ADAHOP_OK)
        rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void *>(&k_wgrad8<2, 2>), hipFuncAttributeMaxDynamicSharedMemorySize, tile_t<2, 2>::LDS));
    if (rc == ADAHOP_OK) g_once.mark(dev);
    return rc;
}

size_t wgrad8_workspace_bytes(int64_t T, int64_t N, int64_t D)
{
    const plan_t p = plan_of(T, N, D);
    return p.slices > 1 ? (size_t)p.slices * N * D * sizeof(float) : 0;
}

int launch_wgrad8(int64_t T, int64_t N, int64_t D, const adahop_tensor_t &G, const adahop_ckpt8_t &x, const adahop_tensor_t &col_scale,
                  const adahop_tensor_t &add, const adahop_tensor_t &C, void *workspace, hipStream_t st)
{
    int rc = configure_wgrad8();
    if (rc != ADAHOP_OK) return rc;
    const plan_t p = plan_of(T, N, D);
    wgrad_t q = {G, col_scale, add, C, x, T, N, D, p.slices > 1 ? static_cast<float *>(workspace) : nullptr, p.slice, 0, 0};
    if (p.large) {
        q.nt = (uint32_t)ceil_div(N, 256), q.dt = (uint32_t)ceil_div(D, 256);
        k_wgrad8<4, 4><<<dim3(q.nt * q.dt, p.slices), 256, tile_t<4, 4>::LDS, st>>>(q);
    } else {
        q.nt = (uint32_t)ceil_div(N, 128), q.dt = (uint32_t)ceil_div(D, 128);
        k_wgrad8<2, 2><<<dim3(q.nt * q.dt, p.slices), 256, tile_t<2, 2>::LDS, st>>>(q);
    }
    rc = check_launch();
    if (rc != ADAHOP_OK || !q.part) return rc;
    k_wgrad8_join<<<dim3((unsigned)ceil_div(D, 256), (unsigned)(N < 65535 ? N : 65535), (unsigned)ceil_div(N, 65535)), 256, 0, st>>>(q, p.slices);
    return check_launch();
}

} // namespace adahop

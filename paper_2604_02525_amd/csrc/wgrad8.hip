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
#include <type_traits>

#include "ckpt8.h"
#include "gemm_mx_common.h"

namespace adahop {

namespace {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));

constexpr int STAGE = 32, STEPS = STAGE / 16; // tokens per stage; matrix-core steps in it

struct wgrad_t {
    adahop_tensor_t G, col_scale, add, C;
    adahop_ckpt8_t x;
    int64_t T, N, D;
    float *part;        // [slices][N][D], or nullptr: one slice, finished by the kernel itself
    int64_t slice;      // tokens per slice, whole stages
    uint32_t nt, dt;    // tiles along N and D
};

// What a workgroup reads: `bytes` from `base` on, below 2^31; beyond that zeros.
__device__ __forceinline__ rsrc_t resource(const uint8_t *base, uint32_t bytes)
{
    base = uniform_ptr(base);
    rsrc_t r;
    r.x = (uint32_t)(uint64_t)base;
    r.y = (uint32_t)((uint64_t)base >> 32);
    r.z = __builtin_amdgcn_readfirstlane(bytes);
    r.w = 0x00027000u;
    return r;
}

// Lane i's 16 bytes (4 bytes) at voff of the resource land at lds + AT + 16 i (4 i); zeros where they lie beyond its end.  (dma16 of gemm_mx_common.h
// with bounds.)  lds: wave-uniform.
template <uint32_t AT> __device__ __forceinline__ void dma16_bounded(rsrc_t r, uint32_t voff, uint32_t lds)
{
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                 :
                 : "v"(voff), "s"(r), "s"(lds), "n"(AT)
                 : "memory", "m0", "scc");
}

// The first LANES <= 32 lanes only, of a wave whose lanes are all active; without a branch, which would end the block that the instructions around
// are scheduled in.
template <uint32_t AT, int LANES> __device__ __forceinline__ void dma4_bounded(rsrc_t r, uint32_t voff, uint32_t lds)
{
    asm volatile("s_add_u32 m0, %2, %3\n\ts_mov_b32 exec_lo, %4\n\ts_mov_b32 exec_hi, 0\n\tbuffer_load_dword %0, %1, 0 offen lds\n\ts_mov_b64 exec, -1"
                 :
                 : "v"(voff), "s"(r), "s"(lds), "n"(AT), "n"((uint32_t)(((uint64_t)1 << LANES) - 1))
                 : "memory", "m0", "scc");
}

__device__ __forceinline__ u32x2 transposed(uint32_t lds_addr)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)lds_addr));
}

__device__ __forceinline__ float element(const adahop_tensor_t &t, int64_t at)
{
    return t.f32 ? static_cast<const float *>(t.data)[at] : bf16_one(static_cast<const uint16_t *>(t.data)[at]);
}

// C[r, c .. c + have) = v times scale, plus what is added.
__device__ __forceinline__ void put4(const adahop_tensor_t &to, const adahop_tensor_t &add, int64_t r, int64_t c, int have, const float (&scale)[4], float4 v)
{
    float o[4] = {v.x * scale[0], v.y * scale[1], v.z * scale[2], v.w * scale[3]};
    if (add.data) {
        const int64_t at = r * add.ld + c;
        if (have == 4 && add.f32) {
            const u32x4 a = *reinterpret_cast<const u32x4_e4 *>(static_cast<const uint32_t *>(add.data) + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] += __uint_as_float(a[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < have) o[i] += element(add, at + i);
        }
    }
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

// Tiles of C by WN x WD waves of 32 MT x 32 NT.  Two waves per SIMD, in one workgroup or in two: a wave issues an instruction every four
// cycles at most, and what it has to issue beside its matrix instructions does not fit between them.
//
// A stage of G (bf16), of X8's codes and of its scales is copied to a ring of RING slots in LDS, RING - 1 stages ahead of its use.  Each
// wave converts the codes that it has copied itself, so that it waits for its own copies alone: it reads those of the stage after the next in the
// second half of a stage, and writes the bf16 rows, into one of two buffers, in the first half of the stage after.  One barrier per stage, in the middle of its
// last step; behind it the first operands of the next stage are read.  The operands of a step are always read during the step before it.  At the
// barrier no wave has reads of the stage at hand outstanding: its buffer is converted to, and its slot copied to, in the next stage.
template <int MT, int NT, int WN, int WD, int RING> struct tile_t {
    static constexpr int WAVES = WN * WD, TM = 32 * WN * MT, TN = 32 * WD * NT, RA = 2 * TM, RB = 2 * TN;      // columns; bytes of a row in LDS
    static constexpr uint32_t A = STAGE * RA, Q = STAGE * TN, S = STAGE * 16, B = STAGE * RB; // bytes of a stage: G, codes, scales, bf16 of X8
    static constexpr uint32_t Q0 = A, S0 = A + Q, SLOT = (S0 + S + 511) / 512 * 512, B0 = RING * SLOT, LDS = B0 + 2 * B; // in a slot: G, codes, scales
    static constexpr int WAVE_ROWS = STAGE / WAVES;                                 // tokens whose codes and scales a wave copies and converts
    static constexpr int COPIES = A / 1024 / WAVES, ROWS_PER_COPY = 1024 / RA;          // of G: per wave and stage
    static constexpr int CODE_COPIES = Q / 1024 / WAVES, ROWS_PER_CODE_COPY = 1024 / TN;
    static constexpr int ISSUED = COPIES + CODE_COPIES + 1;                         // copies per wave and stage
    static constexpr int UNITS = WAVE_ROWS * TN / 8 / 64, ROWS_PER_UNIT = 512 / TN; // of 8 codes per lane
};

// f(i) for i = FROM .. TO - 1, i known at compile time.
template <int FROM, int TO, class F> __device__ __forceinline__ void static_for(F &&f)
{
    if constexpr (FROM < TO) {
        f(std::integral_constant<int, FROM>{});
        static_for<FROM + 1, TO>(f);
    }
}

template <int N> __device__ __forceinline__ void wait_for_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); } // all but the last N

template <int MT, int NT, int WN, int WD, int RING> __global__ __launch_bounds__(64 * WN * WD, 2) void k_wgrad8(wgrad_t q)
{
    typedef tile_t<MT, NT, WN, WD, RING> K;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wn = w / WD, wd = w % WD;
    const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_address(smem));

    // Workgroups go round the eight XCDs; each takes a run of tiles, which it walks in columns of four tiles: what runs on it at a time
    // shares four tiles of G's columns and eight of X's (half as many bytes each).
    const uint32_t tiles = q.nt * q.dt, id = blockIdx.x, per = tiles / 8, rest = tiles % 8, xcd = id % 8;
    const uint32_t t = xcd * per + (xcd < rest ? xcd : rest) + id / 8, group = t / (4 * q.dt), in = t - group * 4 * q.dt;
    const uint32_t high = q.nt - 4 * group < 4 ? q.nt - 4 * group : 4;
    const int64_t n0 = (int64_t)(4 * group + in % high) * K::TM, d0 = (int64_t)(in / high) * K::TN;
    const int64_t begin = (int64_t)blockIdx.y * q.slice, end = begin + q.slice < q.T ? begin + q.slice : q.T;

    // What this wave and this lane copy of a stage.
    const uint32_t ld = (uint32_t)(q.G.ld * 2), ldc = (uint32_t)q.x.ld_codes, lds_s = (uint32_t)q.x.ld_scales;
    uint32_t voff[K::COPIES], qoff[K::CODE_COPIES];
#pragma unroll
    for (int i = 0; i < K::COPIES; ++i) {
        const uint32_t row = (w * K::COPIES + i) * K::ROWS_PER_COPY + lane / (K::RA / 16), chunk = lane % (K::RA / 16);
        voff[i] = row * ld + (((chunk >> 2) ^ (row & 3)) * 64 + (chunk & 3) * 16);
    }
#pragma unroll
    for (int i = 0; i < K::CODE_COPIES; ++i) qoff[i] = ((w * K::CODE_COPIES + i) * K::ROWS_PER_CODE_COPY + lane / (K::TN / 16)) * ldc + lane % (K::TN / 16) * 16;
    // Scales: at most eight bytes of a row, at any address: four whole words from the one on that holds the first.
    const uint8_t *sp = q.x.scales + begin * q.x.ld_scales + (d0 >> 5);
    const uint32_t odd = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)sp & 3); // the same in every stage
    const uint32_t soff = ((odd + (w * K::WAVE_ROWS + lane / 4) * lds_s) & ~3u) + lane % 4 * 4;
    // bytes of `rows` rows of a stage that exist, in whole words
    const auto extent = [&](uint32_t rows, uint32_t pitch, int64_t last, int64_t most) {
        return rows ? ((rows - 1) * pitch + (uint32_t)(last < most ? last : most) + 3) & ~3u : 0u;
    };
    const int64_t ge = (q.N - n0) * 2, xe = q.D - d0, se = odd + ((q.D - d0 + 31) >> 5);
    const uint32_t gfull = extent(STAGE, ld, ge, K::RA), xfull = extent(STAGE, ldc, xe, K::TN), sfull = extent(STAGE, lds_s, se, 16);
    rsrc_t rg = resource(reinterpret_cast<const uint8_t *>(q.G.data) + begin * q.G.ld * 2 + n0 * 2, gfull);
    rsrc_t rx = resource(q.x.codes + begin * q.x.ld_codes + d0, xfull), rs = resource(sp - odd, sfull);
    int32_t ahead = (int32_t)(end - begin), left = ahead; // tokens from the stage that is copied next on, and from the one at hand on
    const uint32_t base = lds;
    uint32_t to = base, raw = base, at = base; // slots: copied to next, whose codes are read next, whose operands are
    uint32_t buffer = base + K::B0;            // of the converted rows
    const auto after = [&](uint32_t slot) { return slot == base + (RING - 1) * K::SLOT ? base : slot + K::SLOT; };
    const auto trim = [&] { // the resources of the stage that is copied next, where it is not a whole one
        if (ahead >= STAGE) return;
        const uint32_t rows = ahead > 0 ? (uint32_t)ahead : 0;
        rg.z = extent(rows, ld, ge, K::RA);
        rx.z = extent(rows, ldc, xe, K::TN);
        rs.z = extent(rows, lds_s, se, 16);
    };
    const auto forward = [](rsrc_t &r, uint32_t bytes) {
        const uint64_t p = ((uint64_t)r.y << 32 | r.x) + bytes;
        r.x = (uint32_t)p;
        r.y = (uint32_t)(p >> 32);
    };
    const uint32_t gstep = STAGE * ld, xstep = STAGE * ldc, sstep = STAGE * lds_s;
    const auto copied = [&] {
        forward(rg, gstep);
        forward(rx, xstep);
        forward(rs, sstep);
        ahead -= STAGE;
        to = after(to);
    };
    const uint32_t own_g = w * K::COPIES * 1024, own_q = w * K::CODE_COPIES * 1024, own_s = w * K::WAVE_ROWS * 16;
    const auto copy = [&](auto number) {
        constexpr int i = decltype(number)::value;
        if constexpr (i < K::COPIES)
            dma16_bounded<i * 1024>(rg, voff[i], to + own_g);
        else if constexpr (i < K::COPIES + K::CODE_COPIES)
            dma16_bounded<K::Q0 + (i - K::COPIES) * 1024>(rx, qoff[i - K::COPIES], to + own_q);
        else
            dma4_bounded<K::S0, 4 * K::WAVE_ROWS>(rs, soff, to + own_s);
    };

    // What it converts and reads.
    const uint32_t urow = w * K::WAVE_ROWS + lane / (K::TN / 8), unit = lane % (K::TN / 8);
    const uint32_t raw_at = K::Q0 + w * K::WAVE_ROWS * K::TN + lane * 8;
    uint32_t scale_at[K::UNITS], put[K::UNITS];
#pragma unroll
    for (int j = 0; j < K::UNITS; ++j) {
        const uint32_t r = urow + j * K::ROWS_PER_UNIT;
        scale_at[j] = K::S0 + r * 16 + ((odd + r * lds_s) & 3) + unit / 4;
        put[j] = r * K::RB + (((unit >> 2) ^ (r & 3)) * 64 + (unit & 3) * 16);
    }
    const int s16 = lane & 15, h = lane >> 5;
    uint32_t ra[MT], rb[NT], va[MT], vb[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) ra[m] = (8 * h + (s16 >> 2)) * K::RA + (((wn * MT + m) ^ (s16 >> 2)) * 64) + 32 * ((lane >> 4) & 1) + 8 * (s16 & 3);
#pragma unroll
    for (int n = 0; n < NT; ++n) rb[n] = (8 * h + (s16 >> 2)) * K::RB + (((wd * NT + n) ^ (s16 >> 2)) * 64) + 32 * ((lane >> 4) & 1) + 8 * (s16 & 3);
    u32x2 codes[K::UNITS];
    uint32_t scales[K::UNITS];
    const auto fetch = [&](int j) {
        codes[j] = *(__attribute__((address_space(3))) u32x2 *)(raw + raw_at + j * 512);
        scales[j] = *(__attribute__((address_space(3))) uint8_t *)(raw + scale_at[j]);
    };
    const auto convert = [&](int j) {
        const float scale = __uint_as_float(scales[j] << 23);
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[j][i], scale, false));
            v[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[j][i], scale, true));
        }
        *(__attribute__((address_space(3))) u32x4 *)(buffer + put[j]) = v;
    };

    v16f acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = {};
    u32x2 fa[2][MT][2], fb[2][NT][2];
    // Read number i of a step's operands, in the order in which they are used: G's first tile, all of X's, G's others.  The first step's
    // go to the stage whose slot and buffer are at hand.
    const auto read = [&](int step, int i) {
        const int tile = i >> 1, part = i & 1;
        if (tile >= 1 && tile <= NT) {
            if (step == 0 && part == 0) vb[tile - 1] = buffer + rb[tile - 1];
            fb[step][tile - 1][part] = transposed(vb[tile - 1] + (16 * step + 4 * part) * K::RB);
        } else {
            const int m = tile ? tile - NT : 0;
            if (step == 0 && part == 0) va[m] = at + ra[m];
            fa[step][m][part] = transposed(va[m] + (16 * step + 4 * part) * K::RA);
        }
    };
    // A step's matrix instructions are places, with what is issued beside each.  Step 0: conversions, and all reads of step 1; step 1: the barrier
    // beside place BARRIER, behind it reads and codes.  The copies are spread over both steps.
    constexpr int READS = 2 * (MT + NT), PLACES = MT * NT, BARRIER = PLACES / 2 - 1, FETCH = BARRIER + 1, EARLY = PLACES - PLACES / 4;
    constexpr auto copy_at = [](int i) { return (2 * i + 1) * PLACES / K::ISSUED; }; // of 2 PLACES
    constexpr auto copies_before = [](int place) {
        int n = 0;
        while (n < K::ISSUED && (2 * n + 1) * PLACES / K::ISSUED < place) ++n;
        return n;
    };
    static_assert(STEPS == 2 && K::UNITS <= PLACES - FETCH && K::UNITS <= PLACES, "a stage's work fits its two steps");
    const auto other = [&](uint32_t b) { return b == base + K::B0 ? base + K::B0 + K::B : base + K::B0; };

    if (left > 0) {
#pragma unroll 1
        for (int i = 0; i < RING - 1; ++i) {
            trim();
            static_for<0, K::ISSUED>(copy);
            copied();
        }
        trim();
        wait_for_copies<(RING - 2) * K::ISSUED>();
#pragma unroll
        for (int j = 0; j < K::UNITS; ++j) fetch(j);
#pragma unroll
        for (int j = 0; j < K::UNITS; ++j) convert(j);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        raw = after(raw);
        wait_for_copies<(RING - 3) * K::ISSUED>();
#pragma unroll
        for (int j = 0; j < K::UNITS; ++j) fetch(j); // first, as in the loop: the compiler's waits go by how many reads may be behind these
        ADAHOP_PIN();
#pragma unroll
        for (int i = 0; i < READS; ++i) read(0, i);
    }
    while (left > 0) {
        static_for<0, 2 * PLACES>([&](auto number) {
            constexpr int all = decltype(number)::value, step = all / PLACES, place = all % PLACES, m = place / NT, n = place % NT;
            const auto whole = [](const u32x2 (&f)[2]) { return make_uint4(f[0].x, f[0].y, f[1].x, f[1].y); };
            acc[m][n] = mfma_bf16(whole(fa[step][m]), whole(fb[step][n]), acc[m][n]);
            if constexpr (step == 0) {
                if constexpr (place == 0) buffer = other(buffer);
                if constexpr (place < K::UNITS) convert(place);
#pragma unroll
                for (int i = place * READS / EARLY; i < (place + 1) * READS / EARLY && i < READS; ++i) read(1, i);
            } else if constexpr (place == BARRIER) {
                at = raw;
                raw = after(raw);
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            } else if constexpr (place > BARRIER) {
                constexpr int LEFT = PLACES - 1 - BARRIER, behind = place - 1 - BARRIER;
#pragma unroll
                for (int i = behind * READS / LEFT; i < (behind + 1) * READS / LEFT; ++i) read(0, i);
                // the codes of the stage after the next: all copies but those of the stage behind it and what this stage has issued so far are done
                if constexpr (place == FETCH) wait_for_copies<(RING - 4) * K::ISSUED + copies_before(all)>();
                if constexpr (place >= FETCH && place < FETCH + K::UNITS) fetch(place - FETCH);
            }
            static_for<0, K::ISSUED>([&](auto i) {
                if constexpr (copy_at(decltype(i)::value) == all) copy(i);
            });
            ADAHOP_PIN();
        });
        copied();
        trim();
        left -= STAGE;
    }

    // C, 32 rows of a wave at a time by way of its own patch of LDS, so that a lane has four consecutive columns of a row: 16-byte stores of
    // whole rows, and little code.  In the accumulators a lane has column lane % 32 of a tile, rows 8 (i / 4) + 4 h + i % 4.
    wait_for_copies<0>();
    asm volatile("s_barrier" ::: "memory"); // no wave reads or copies any more
    constexpr int PITCH = 32 * NT + 4, LANES = 8 * NT;
    float *const patch = reinterpret_cast<float *>(smem) + w * 32 * PITCH;
    const int c4 = lane % LANES * 4, r0 = lane / LANES;
    const int64_t c = d0 + wd * NT * 32 + c4;
    const int have = (int)(q.D - c < 4 ? q.D - c : 4);
    float scale[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    if (q.col_scale.data) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) scale[i] = element(q.col_scale, c + i);
    }
    adahop_tensor_t result = q.C;
    if (q.part) result = {q.part + (int64_t)blockIdx.y * q.N * q.D, q.D, 1};
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        lds_between_lanes();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) patch[(8 * (i >> 2) + 4 * h + (i & 3)) * PITCH + 32 * n + (lane & 31)] = acc[m][n][i];
        lds_between_lanes();
        const int64_t first = n0 + (wn * MT + m) * 32 + r0;
        if (have <= 0) continue;
#pragma unroll 4
        for (int i = 0; i < 32; i += 64 / LANES) {
            const int64_t r = first + i;
            if (r < q.N) put4(result, q.add, r, c, have, scale, *reinterpret_cast<const float4 *>(patch + (r0 + i) * PITCH + c4));
        }
    }
}

// The sums of the slices, in their order, and what the kernel above does with a single one's.  A lane has four columns.
__global__ __launch_bounds__(256) void k_wgrad8_join(wgrad_t q, int slices)
{
    const int64_t c = ((int64_t)blockIdx.x * 64 + (threadIdx.x & 63)) * 4, r = (int64_t)blockIdx.y * 4 + (threadIdx.x >> 6);
    if (c >= q.D || r >= q.N) return;
    const int have = (int)(q.D - c < 4 ? q.D - c : 4);
    float v[4] = {}, scale[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    const uint32_t *p = reinterpret_cast<const uint32_t *>(q.part) + r * q.D + c;
    if (have == 4) {
#pragma unroll 4
        for (int s = 0; s < slices; ++s, p += q.N * q.D) {
            const u32x4 a = *reinterpret_cast<const u32x4_e4 *>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += __uint_as_float(a[i]);
        }
    } else {
        for (int s = 0; s < slices; ++s, p += q.N * q.D)
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < have) v[i] += __uint_as_float(p[i]);
    }
    if (q.col_scale.data) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) scale[i] = element(q.col_scale, c + i);
    }
    put4(q.C, q.add, r, c, have, scale, make_float4(v[0], v[1], v[2], v[3]));
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
    rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void *>(&k_wgrad8<4, 2, 2, 4, 5>), hipFuncAttributeMaxDynamicSharedMemorySize, tile_t<4, 2, 2, 4, 5>::LDS));
    if (rc == ADAHOP_OK)
        rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void *>(&k_wgrad8<2, 2, 2, 2, 5>), hipFuncAttributeMaxDynamicSharedMemorySize, tile_t<2, 2, 2, 2, 5>::LDS));
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
    if (q.part) q.col_scale = q.add = {}; // the slices' sums come first
    if (p.large) {
        q.nt = (uint32_t)ceil_div(N, 256), q.dt = (uint32_t)ceil_div(D, 256);
        k_wgrad8<4, 2, 2, 4, 5><<<dim3(q.nt * q.dt, p.slices), 512, tile_t<4, 2, 2, 4, 5>::LDS, st>>>(q);
    } else {
        q.nt = (uint32_t)ceil_div(N, 128), q.dt = (uint32_t)ceil_div(D, 128);
        k_wgrad8<2, 2, 2, 2, 5><<<dim3(q.nt * q.dt, p.slices), 256, tile_t<2, 2, 2, 2, 5>::LDS, st>>>(q);
    }
    rc = check_launch();
    if (rc != ADAHOP_OK || !q.part) return rc;
    q.col_scale = col_scale, q.add = add;
    k_wgrad8_join<<<dim3((unsigned)ceil_div(D, 256), (unsigned)ceil_div(N, 4)), 256, 0, st>>>(q, p.slices);
    return check_launch();
}

} // namespace adahop

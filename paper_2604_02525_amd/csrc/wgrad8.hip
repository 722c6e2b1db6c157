// Weight gradient of a linear layer from the 8-bit checkpoint of its input (paper Eq. 3 with X kept in 8 bits):
//
//     C[n, d] = w[d] sum_t G[t, n] X8[t, d] (+ add[n, d])
//
// on the BF16 matrix cores: an E4M3 element times its power of two is a bf16 number, so nothing is rounded on the way there.  The checkpoint is expanded
// to bf16 rows in the workspace (3 bytes per element moved), then both operands are bf16.  For 28672 columns of G the expansion is 1.2 % of the time, for 4096
// 8 %.  Converting in the product itself takes longer: codes converted once per workgroup, by way of LDS, took 6.4 ms at 16384 x 28672 x 8192
// (writing 1024 bytes to LDS takes 13 cycles, reading them 4), in the registers of each wave that needs them 6.9 ms; this takes 5.4 ms.
//
// Bound by the matrix cores and the power that they draw: the product runs at 1.44 PFLOP/s with the clock down to 1.78 GHz (2.4 GHz on operands of
// zeros), a library product of operands that have the contraction contiguous at 1.58.  The 16 x 16 x 32 instructions draw less than those of 32 x 32 x 16
// (alone, on random operands, 2.06 against 1.85 PFLOP/s).
//
// Both operands have the contraction (tokens) along their rows, the matrix cores want it within a lane: the transposing read of LDS
// (ds_read_b64_tr_b16) turns them, four tokens of a column per lane and read, at the rate of plain reads.  They go to LDS as they are, by copies that pass no
// register (16 bytes per lane).  Rows past the last token read as zero (the bounds of a buffer resource), in both operands: infinities and NaN meet
// no padding.  Columns past the operands' hold whatever is there; they end in elements of C that are not stored.
//
// LDS layout: token t's row at t * row bytes, its pieces of 32 bytes (the columns of one matrix-core operand) exchanged by t's bits 0, 1 and 3: the eight
// rows that a transposing read of half a wave touches lie in eight different eighths of the banks.
#include <type_traits>

#include "ckpt8.h"
#include "gemm_mx_common.h"

namespace adahop {

namespace {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));

constexpr int STAGE = 32; // tokens per stage: one matrix instruction's

struct wgrad_t {
    adahop_tensor_t G, X, col_scale, add, C;
    int64_t T, N, D;
    float *part;        // [slices][N][D], or nullptr: one slice, finished by the kernel itself
    int64_t slice;      // tokens per slice, whole stages
    uint32_t nt, dt;    // tiles along N and D
};

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

// Tiles of C by WN x WD waves of 16 MT x 16 NT.  Two waves per SIMD, in one workgroup or in two: a wave issues an instruction every four cycles at
// most, too few for one to feed the matrix cores and LDS.
//
// A stage of both operands is copied to a ring of RING slots in LDS, RING - 1 stages ahead of its use.  A wave's operands of G are read again, for the
// next stage, behind the last of the NT matrix instructions that use them, those of X into a second set of registers.  SPLIT = 2: two shares of such waves,
// each with half of the tokens and a ring of its own, whose sums meet at the end.  One barrier per stage, behind the
// first NT instructions: what is read after it has been copied by all waves, and nothing of the stage before is still to be read, so that its slot
// is copied to, at the end of the stage (earlier: 2 % slower).
template <int MT, int NT, int WN, int WD, int RING, int SPLIT = 1> struct tile_t {
    static constexpr int WAVES = WN * WD, THREADS = 64 * WAVES * SPLIT, TM = 16 * WN * MT, TN = 16 * WD * NT, RA = 2 * TM, RB = 2 * TN; // columns; bytes of a row in LDS
    static constexpr uint32_t A = STAGE * RA, B = STAGE * RB, SLOT = A + B, LDS = SPLIT * RING * SLOT;
    static constexpr int COPIES_A = A / 1024 / WAVES, COPIES_B = B / 1024 / WAVES, ISSUED = COPIES_A + COPIES_B; // per wave and stage
    static __device__ __forceinline__ uint32_t turn_of(uint32_t row) { return (row & 3) | (row >> 1 & 4); }      // of the pieces of a row
    // What lane l of copy number `copy` of a stage reads: its row, and the byte in it
    static __device__ __forceinline__ uint32_t row_of(uint32_t copy, uint32_t l, uint32_t bytes) { return (copy * 1024 + l * 16) / bytes; }
    static __device__ __forceinline__ uint32_t byte_of(uint32_t row, uint32_t l, uint32_t bytes)
    {
        const uint32_t chunk = l % (bytes / 16);
        return ((chunk >> 1) ^ turn_of(row)) * 32 + (chunk & 1) * 16;
    }
};

template <int MT, int NT, int WN, int WD, int RING, int SPLIT> __global__ __launch_bounds__(64 * WN * WD * SPLIT, 2) void k_wgrad8(wgrad_t q)
{
    typedef tile_t<MT, NT, WN, WD, RING, SPLIT> K;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), share = SPLIT > 1 ? wave / K::WAVES : 0;
    const int w = wave - share * K::WAVES, wn = w / WD, wd = w % WD;
    const uint32_t base = __builtin_amdgcn_readfirstlane(lds_address(smem)) + share * RING * K::SLOT;

    // Workgroups go round the eight XCDs; each takes a run of tiles, which it walks in columns of four tiles: what runs on it at a time
    // shares few tiles of either operand.
    const uint32_t tiles = q.nt * q.dt, id = blockIdx.x, per = tiles / 8, rest = tiles % 8, xcd = id % 8;
    const uint32_t t = xcd * per + (xcd < rest ? xcd : rest) + id / 8, group = t / (4 * q.dt), in = t - group * 4 * q.dt;
    const uint32_t high = q.nt - 4 * group < 4 ? q.nt - 4 * group : 4;
    const int64_t n0 = (int64_t)(4 * group + in % high) * K::TM, d0 = (int64_t)(in / high) * K::TN;
    int64_t begin = (int64_t)blockIdx.y * q.slice, end = begin + q.slice < q.T ? begin + q.slice : q.T;
    int32_t left = (int32_t)(end - begin); // tokens from the stage at hand on, of the first share
    if constexpr (SPLIT > 1) {             // this wave's share of them, whole pairs of stages; the last may have none
        const int32_t each = (left + 2 * SPLIT * STAGE - 1) / (2 * SPLIT * STAGE) * (2 * STAGE);
        begin += (int64_t)share * each;
        end = begin + each < end ? begin + each : end < begin ? begin : end;
        left = left < each ? left : each;
    }

    // What this wave and this lane copy of a stage.
    const uint32_t lda = (uint32_t)(q.G.ld * 2), ldb = (uint32_t)(q.X.ld * 2);
    uint32_t aoff[K::COPIES_A], boff[K::COPIES_B];
#pragma unroll
    for (int i = 0; i < K::COPIES_A; ++i) {
        const uint32_t row = K::row_of(w * K::COPIES_A + i, lane, K::RA);
        aoff[i] = row * lda + K::byte_of(row, lane, K::RA);
    }
#pragma unroll
    for (int i = 0; i < K::COPIES_B; ++i) {
        const uint32_t row = K::row_of(w * K::COPIES_B + i, lane, K::RB);
        boff[i] = row * ldb + K::byte_of(row, lane, K::RB);
    }
    // bytes of `rows` rows of a stage that exist, in whole words
    const auto extent = [](uint32_t rows, uint32_t pitch, int64_t last, int64_t most) {
        return rows ? ((rows - 1) * pitch + (uint32_t)(last < most ? last : most) + 3) & ~3u : 0u;
    };
    const uint32_t odd_rows = (uint32_t)(end - begin) % STAGE;
    const uint32_t afull = extent(STAGE, lda, (q.N - n0) * 2, K::RA), alast = extent(odd_rows, lda, (q.N - n0) * 2, K::RA);
    const uint32_t bfull = extent(STAGE, ldb, (q.D - d0) * 2, K::RB), blast = extent(odd_rows, ldb, (q.D - d0) * 2, K::RB);
    rsrc_t from_a = resource(static_cast<const uint16_t *>(q.G.data) + begin * q.G.ld + n0, afull);
    rsrc_t from_b = resource(static_cast<const uint16_t *>(q.X.data) + begin * q.X.ld + d0, bfull);
    int32_t ahead = (int32_t)(end - begin); // tokens from the stage that is copied next on
    uint32_t to = base, at = base;          // slots: copied to next, read next
    const auto after = [&](uint32_t slot) { return slot == base + (RING - 1) * K::SLOT ? base : slot + K::SLOT; };
    const auto forward = [](rsrc_t &r, uint32_t bytes) {
        const uint64_t p = ((uint64_t)r.y << 32 | r.x) + bytes;
        r.x = (uint32_t)p;
        r.y = (uint32_t)(p >> 32);
    };
    // The resources of the stage that is copied next: a whole one, the last rows, or nothing.  Without a branch: it would end the block that the
    // instructions around are scheduled in.
    const auto trim = [&] {
        from_a.z = ahead >= STAGE ? afull : ahead > 0 ? alast : 0;
        from_b.z = ahead >= STAGE ? bfull : ahead > 0 ? blast : 0;
    };
    const uint32_t step_a = STAGE * lda, step_b = STAGE * ldb, own_a = w * K::COPIES_A * 1024, own_b = w * K::COPIES_B * 1024;
    const auto copied = [&] {
        forward(from_a, step_a);
        forward(from_b, step_b);
        ahead -= STAGE;
        to = after(to);
        trim();
    };
    const auto copy = [&](auto number) {
        constexpr int i = decltype(number)::value;
        if constexpr (i < K::COPIES_A)
            dma16_bounded<i * 1024>(from_a, aoff[i], to + own_a);
        else
            dma16_bounded<K::A + (i - K::COPIES_A) * 1024>(from_b, boff[i - K::COPIES_A], to + own_b);
    };

    // What it reads: the matrix instruction wants the eight tokens from 8 (lane / 16) on of column lane % 16.  Four lanes of a group of 16 supply the
    // four pieces of a row, of four columns each; the group receives four rows.
    const int s16 = lane & 15, g = lane >> 4;
    uint32_t ra[MT], rb[NT];
#pragma unroll
    for (int m = 0; m < MT; ++m) ra[m] = (8 * g + (s16 >> 2)) * K::RA + (((wn * MT + m) ^ K::turn_of(8 * g + (s16 >> 2))) * 32) + 8 * (s16 & 3);
#pragma unroll
    for (int n = 0; n < NT; ++n) rb[n] = K::A + (8 * g + (s16 >> 2)) * K::RB + (((wd * NT + n) ^ K::turn_of(8 * g + (s16 >> 2))) * 32) + 8 * (s16 & 3);
    v4f acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = {};
    u32x2 fa[MT][2], fb[2][NT][2];
    uint32_t lies = 0;
    const auto read_a = [&](int m, int part) {
        if (!part) lies = at + ra[m];
        fa[m][part] = transposed(lies + 4 * part * K::RA);
    };
    const auto read_b = [&](int set, int n, int part) {
        if (!part) lies = at + rb[n];
        fb[set][n][part] = transposed(lies + 4 * part * K::RB);
    };
    constexpr int PLACES = MT * NT, BARRIER = NT - 1; // a stage's matrix instructions are places, with what is issued beside each
    constexpr int EACH = (2 * NT + (MT - 1) * (NT - 2) - 1) / ((MT - 1) * (NT - 2)); // reads of X's operands beside one of the places for them
    static_assert(NT > 2 && K::ISSUED <= PLACES - NT, "what goes beside the matrix instructions fits");

    trim();
#pragma unroll 1
    for (int i = 0; i < RING - 1; ++i) {
        static_for<0, K::ISSUED>(copy);
        copied();
    }
    wait_for_copies<(RING - 2) * K::ISSUED>();
    // Everything that the compiler counts with the reads of LDS is done before these, and these are issued in the order of the loop's: its waits in
    // the loop go by what may be outstanding on either way into it.
    __builtin_amdgcn_s_waitcnt(0xc07f); // lgkmcnt(0)
    asm volatile("s_barrier" ::: "memory");
    ADAHOP_PIN();
#pragma unroll
    for (int n = 0; n < NT; ++n) read_b(0, n, 0), read_b(0, n, 1);
#pragma unroll
    for (int m = 0; m < MT - 1; ++m) {
        ADAHOP_PIN();
        read_a(m, 0), read_a(m, 1);
    }
    ADAHOP_PIN();
    const auto stage = [&](auto which) {
        constexpr int set = decltype(which)::value;
        static_for<0, PLACES>([&](auto number) {
            constexpr int place = decltype(number)::value, m = place / NT, n = place % NT;
            const uint4 a = make_uint4(fa[m][0].x, fa[m][0].y, fa[m][1].x, fa[m][1].y);
            const uint4 b = make_uint4(fb[set][n][0].x, fb[set][n][0].y, fb[set][n][1].x, fb[set][n][1].y);
            acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), acc[m][n], 0, 0, 0);
            if constexpr (m == 0 && n < 2) read_a(MT - 1, n); // of this stage
            if constexpr (place == BARRIER) {
                asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((RING - 3) * K::ISSUED) : "memory"); // the next stage is there
                at = after(at);
            }
            if constexpr (m > 0) {
                constexpr int first = ((m - 1) * (NT - 2) + n - 2) * EACH;
                if constexpr (n < 2)
                    read_a(m - 1, n);
                else
                    static_for<first, first + EACH < 2 * NT ? first + EACH : 2 * NT>([&](auto i) { read_b(set ^ 1, decltype(i)::value >> 1, decltype(i)::value & 1); });
            }
            if constexpr (place >= PLACES - K::ISSUED) copy(std::integral_constant<int, place - (PLACES - K::ISSUED)>{});
            ADAHOP_PIN();
        });
        copied();
        left -= STAGE;
    };
    while (left > 0) { // two stages, one of each set of X's registers; the second may be one of zeros
        stage(std::integral_constant<int, 0>{});
        stage(std::integral_constant<int, 1>{});
    }

    // C, 32 rows of a wave at a time by way of its own patch of LDS, so that a lane has four consecutive columns of a row: 16-byte stores of
    // whole rows, and little code.  In the accumulators a lane has column lane % 16 of a tile, rows 4 (lane / 16) + i.  What is added is read 32 rows
    // ahead: no load passes a store that it might depend on (8192 tokens of 4096 x 4096, added to: 228 us, without 238).
    constexpr int PITCH = 16 * NT + 4, LANES = 4 * NT, STEPS = LANES / 2;
    const int c4 = lane % LANES * 4, r0 = lane / LANES;
    const int64_t c = d0 + wd * NT * 16 + c4;
    const int have = (int)(q.D - c < 4 ? q.D - c : 4);
    const auto row_at = [&](int m, int i) { return n0 + (wn * MT + m) * 16 + r0 + i * (64 / LANES); };
    float scale[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    if (q.col_scale.data) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) scale[i] = element(q.col_scale, c + i);
    }
    float *const patch = reinterpret_cast<float *>(smem) + wave * 32 * PITCH;
    adahop_tensor_t result = q.C;
    if (q.part) result = {q.part + (int64_t)blockIdx.y * q.N * q.D, q.D, 1};
    const auto finish = [&](auto adds, auto from, auto till) { // the accumulators' rows `from` to `till`
        constexpr bool ADDS = decltype(adds)::value;
        constexpr int FROM = decltype(from)::value, TILL = decltype(till)::value;
        float4 more[2][STEPS];
        const auto get = [&](int m) {
#pragma unroll
            for (int i = 0; i < STEPS; ++i)
                more[m / 2 & 1][i] = have > 0 && row_at(m, i) < q.N ? get4(q.add, row_at(m, i), c, have) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        };
        if constexpr (ADDS) get(FROM);
        wait_for_copies<0>();
        asm volatile("s_barrier" ::: "memory"); // no wave reads or copies any more
        if constexpr (SPLIT > 1) {              // the other share's sums of these rows, for its sums of the other rows
            constexpr int OTHER = FROM ? 0 : MT / 2;
            v4f *const box = reinterpret_cast<v4f *>(smem) + w * 64 + lane;
            const auto place = [&](int of, int m, int n) -> v4f & { return box[((of * MT / 2 + m) * NT + n) * K::WAVES * 64]; };
#pragma unroll
            for (int m = 0; m < MT / 2; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) place(share, m, n) = acc[OTHER + m][n];
            __syncthreads();
#pragma unroll
            for (int m = 0; m < MT / 2; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[FROM + m][n] += place(1 - share, m, n);
            __syncthreads();
        }
#pragma unroll
        for (int m = FROM; m < TILL; m += 2) {
            lds_between_lanes();
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 8; ++i) patch[(16 * (i >> 2) + 4 * (lane >> 4) + (i & 3)) * PITCH + 16 * n + (lane & 15)] = acc[m + (i >> 2)][n][i & 3];
            lds_between_lanes();
            if (have <= 0) continue;
            if constexpr (ADDS) {
                if (m + 2 < TILL) get(m + 2);
            }
#pragma unroll(ADDS ? STEPS : 4)
            for (int i = 0; i < STEPS; ++i)
                if (row_at(m, i) < q.N)
                    put4(result, row_at(m, i), c, have, scale, *reinterpret_cast<const float4 *>(patch + (r0 + i * (64 / LANES)) * PITCH + c4),
                         ADDS ? more[m / 2 & 1][i] : make_float4(0.0f, 0.0f, 0.0f, 0.0f));
        }
    };
    const auto finish_rows = [&](auto from, auto till) { q.add.data ? finish(std::true_type{}, from, till) : finish(std::false_type{}, from, till); };
    if constexpr (SPLIT == 1) {
        finish_rows(std::integral_constant<int, 0>{}, std::integral_constant<int, MT>{});
    } else {
        static_assert(SPLIT == 2 && MT % 4 == 0, "each share finishes half of the rows");
        if (share == 0)
            finish_rows(std::integral_constant<int, 0>{}, std::integral_constant<int, MT / 2>{});
        else
            finish_rows(std::integral_constant<int, MT / 2>{}, std::integral_constant<int, MT>{});
    }
}

// The sums of the slices, in their order, and what the kernel above does with a single one's.  A lane has four columns.
__global__ __launch_bounds__(256) void k_wgrad8_join(wgrad_t q, int slices)
{
    const int64_t c = ((int64_t)blockIdx.y * 64 + (threadIdx.x & 63)) * 4, r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
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
    put4(q.C, r, c, have, scale, make_float4(v[0], v[1], v[2], v[3]), get4(q.add, r, c, have));
}

struct plan_t {
    bool large;     // tiles of 256 x 256, else 128 x 128
    bool alone;     // one workgroup at most per compute unit
    int slices;
    int64_t slice, ldx;
    size_t part_at, bytes;
};

// Tile size and slices of the tokens by expected time, in microseconds, measured on 256 compute units.  A stage of a round of workgroups: 0.7 with the large
// tiles, one workgroup per compute unit; with the small ones 0.5 where there are two per compute unit, 0.3 where there is one; a round's beginning and end
// 4 and 2.5.  Slices cost their sums' way to memory and back and one launch more.  Both sides at 2048 x 2048, us: 1001 tokens, small tiles in one slice 20.4, in two
// 28.3, large ones in four 36.4; 8192 tokens 72, 78 and 80, 16384 tokens 162, 174 and 132; 4096 tokens of 4096 x 2048, small 67, large in two slices 75, at 16384
// tokens 308 and 220; 16384 tokens of 1024 x 1024, small in one, two and four slices 101, 63 and 49.
//
// Where no compute unit has two workgroups, one of small tiles has two shares of four waves, each with half of the tokens: 1001 tokens of 2048 x 2048 in 20.4 us, with one
// share 22.9 (eight waves on one tile, with half as many matrix instructions for an operand read, 21.2), 2048 tokens 28.5, with one share 33.
plan_t plan_of(int64_t T, int64_t N, int64_t D)
{
    const int64_t stages = ceil_div(T, STAGE), large = ceil_div(N, 256) * ceil_div(D, 256), small = ceil_div(N, 128) * ceil_div(D, 128);
    plan_t p;
    double best = 0.0;
    p.slices = 0;
    for (int64_t slices = 1; slices <= 64 && (slices == 1 || stages / slices >= 8); ++slices) {
        const int64_t each = ceil_div(ceil_div(stages, slices), 2) * 2; // stages per slice; the kernel takes them in pairs
        const int64_t number = T > 0 ? ceil_div(stages, each) : 1;
        const double join = number > 1 ? 6.0 + (double)number * N * D * 8 / 5e6 : 0.0;
        const int64_t rounds = small * number / 512, over = small * number % 512;
        const double in_large = ceil_div(large * number, 256) * (4.0 + 0.7 * each) + join;
        const double in_small = (rounds + (over > 0)) * 2.5 + (rounds * 0.5 + (over > 256 ? 0.5 : over > 0 ? 0.3 : 0.0)) * each + join;
        const double t = in_large < in_small ? in_large : in_small;
        if (p.slices == 0 || t < best) {
            best = t;
            p.large = in_large < in_small;
            p.alone = small * number <= 256;
            p.slices = (int)number;
            p.slice = each * STAGE;
        }
        if (join > best) break;
    }
    p.ldx = ceil_div(D, 8) * 8;
    p.part_at = align_up((size_t)T * p.ldx * 2, 256);
    p.bytes = p.part_at + (p.slices > 1 ? (size_t)p.slices * N * D * sizeof(float) : 0);
    return p;
}

device_once_t g_once;

typedef tile_t<8, 4, 2, 4, 4> large_t;
typedef tile_t<4, 4, 2, 2, 4> small_t;
typedef tile_t<4, 4, 2, 2, 4, 2> small_alone_t;

// tile_t's kernel
template <class K> struct kernel_of;
template <int MT, int NT, int WN, int WD, int RING, int SPLIT> struct kernel_of<tile_t<MT, NT, WN, WD, RING, SPLIT>> {
    typedef tile_t<MT, NT, WN, WD, RING, SPLIT> K;
    static int configure()
    {
        return check_hip(hipFuncSetAttribute(reinterpret_cast<const void *>(&k_wgrad8<MT, NT, WN, WD, RING, SPLIT>), hipFuncAttributeMaxDynamicSharedMemorySize, K::LDS));
    }
    static void launch(wgrad_t &q, int slices, hipStream_t st)
    {
        static_assert(K::THREADS / 64 * 32 * (16 * NT + 4) * sizeof(float) <= K::LDS, "the waves' patches fit");
        static_assert(SPLIT == 1 || 4 * K::TM * K::TN <= K::LDS, "the sums that the shares exchange fit");
        q.nt = (uint32_t)ceil_div(q.N, K::TM), q.dt = (uint32_t)ceil_div(q.D, K::TN);
        k_wgrad8<MT, NT, WN, WD, RING, SPLIT><<<dim3(q.nt * q.dt, slices), K::THREADS, K::LDS, st>>>(q);
    }
};

} // namespace

int configure_wgrad8()
{
    int dev = 0;
    int rc = check_hip(hipGetDevice(&dev));
    if (rc != ADAHOP_OK || !g_once.need(dev)) return rc;
    rc = kernel_of<large_t>::configure();
    if (rc == ADAHOP_OK) rc = kernel_of<small_t>::configure();
    if (rc == ADAHOP_OK) rc = kernel_of<small_alone_t>::configure();
    if (rc == ADAHOP_OK) g_once.mark(dev);
    return rc;
}

size_t wgrad8_workspace_bytes(int64_t T, int64_t N, int64_t D) { return plan_of(T, N, D).bytes; }

void wgrad8_plan(int64_t T, int64_t N, int64_t D, int *tile, int *shares, int *slices)
{
    const plan_t p = plan_of(T, N, D);
    *tile = p.large ? large_t::TM : small_t::TM;
    *shares = !p.large && p.alone ? 2 : 1;
    *slices = p.slices;
}

int launch_wgrad8(int64_t T, int64_t N, int64_t D, const adahop_tensor_t &G, const adahop_ckpt8_t &x, const adahop_tensor_t &col_scale,
                  const adahop_tensor_t &add, const adahop_tensor_t &C, void *workspace, hipStream_t st)
{
    int rc = configure_wgrad8();
    if (rc != ADAHOP_OK) return rc;
    const plan_t p = plan_of(T, N, D);
    const adahop_tensor_t X = {workspace, p.ldx, 0};
    if (T > 0 && (rc = launch_ckpt8_unpack(T, D, x, {}, X, st)) != ADAHOP_OK) return rc;
    float *const part = p.slices > 1 ? reinterpret_cast<float *>(static_cast<char *>(workspace) + p.part_at) : nullptr;
    wgrad_t q = {G, X, col_scale, add, C, T, N, D, part, p.slice, 0, 0};
    if (part) q.col_scale = q.add = {}; // the slices' sums come first
    if (p.large)
        kernel_of<large_t>::launch(q, p.slices, st);
    else if (p.alone)
        kernel_of<small_alone_t>::launch(q, p.slices, st);
    else
        kernel_of<small_t>::launch(q, p.slices, st);
    rc = check_launch();
    if (rc != ADAHOP_OK || !part) return rc;
    q.col_scale = col_scale, q.add = add;
    k_wgrad8_join<<<dim3((unsigned)ceil_div(N, 4), (unsigned)ceil_div(D, 256)), 256, 0, st>>>(q, p.slices);
    return check_launch();
}

} // namespace adahop

// Products of 16-bit operands (bf16 or fp16) on the matrix cores with sums in fp32, for the operators at the end of a training step:
//
//     C[r, c] = sum_k A(r, k) B(c, k)
//
// Either operand may hold the contraction along its rows (ALONG, [outer][K]) or down its columns (DOWN, [K][outer]), so that no operand is ever transposed
// in memory: a gradient of logits [tokens][vocabulary] enters one product by its rows and another by its columns.
//
// The scheme is that of the weight gradient from a checkpoint (wgrad8.hip): both operands go to a ring of stages in LDS by copies that pass no register, 32
// elements of the contraction a stage; a wave's 16 x 16 x 32 instructions are fed from LDS a stage ahead; one barrier per stage.  A DOWN operand is turned by
// the transposing reads of LDS; an ALONG one is read as it lies, 16 bytes (eight elements of a row) per lane.  What lies outside an operand reads as zero, in both.
//
// LDS layout of a stage of an ALONG operand: 64 bytes a row, its four pieces of 16 bytes exchanged by the row's bits 2 and 3: the sixteen rows that a quarter of a wave
// reads one piece of lie in sixteen different sixteenths of the banks.
#pragma once
#include "tile_copies.h"

namespace adahop {

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

enum lies_t { ALONG, DOWN };

struct side_t {
    const uint16_t *data; // 16-byte aligned
    int64_t ld, outer;    // ld: a multiple of 8
};

// Segments: the contraction runs over `segments` products of K elements each, whose operands begin at these elements (an operand held in two halves).
struct segments_t {
    int count;
    int64_t a[3], b[3];
};

struct product_t {
    side_t A, B;
    int64_t K;       // a multiple of 8 where an operand is ALONG; of 32 with several segments
    int64_t slice;   // of all segments' K per slice: a multiple of 64
    float *part;     // [slices][A.outer][B.outer], or nullptr: one slice, finished by the kernel itself
    uint32_t nt, dt; // tiles along A's outer index and B's
    segments_t seg;
    const int32_t *rows_of, *K_of; // (or nullptr) how many of A's outer indices and of the contraction's elements there are, where only the device knows
};

// Tiles of C by WN x WD waves of 16 MT x 16 NT, a ring of RING stages.
template <int MT_, int NT_, int WN_, int WD_, int RING_> struct shape_t {
    static constexpr int MT = MT_, NT = NT_, WN = WN_, WD = WD_, RING = RING_;
    static constexpr int WAVES = WN * WD, THREADS = 64 * WAVES, TM = 16 * WN * MT, TN = 16 * WD * NT, RA = 2 * TM, RB = 2 * TN; // bytes of a row of a DOWN stage
    static constexpr uint32_t A = STAGE * RA, B = STAGE * RB, SLOT = A + B, LDS = RING * SLOT;
    static constexpr int COPIES_A = A / 1024 / WAVES, COPIES_B = B / 1024 / WAVES, ISSUED = COPIES_A + COPIES_B; // per wave and stage
    static_assert(COPIES_A * WAVES * 1024 == A && COPIES_B * WAVES * 1024 == B, "whole copies");
    // DOWN: by what the pieces of 32 bytes of a row are exchanged, so that the eight rows of a transposing read of half a wave lie in different banks
    static __device__ __forceinline__ uint32_t turn_of(uint32_t row, uint32_t bytes) { return bytes >= 256 ? (row & 3) | (row >> 1 & 4) : (row >> 1 & 1) | (row >> 2 & 2); }
    static __device__ __forceinline__ uint32_t row_of(uint32_t copy, uint32_t l, uint32_t bytes) { return (copy * 1024 + l * 16) / bytes; }
    static __device__ __forceinline__ uint32_t byte_of(uint32_t row, uint32_t l, uint32_t bytes)
    {
        const uint32_t chunk = l % (bytes / 16);
        return ((chunk >> 1) ^ turn_of(row, bytes)) * 32 + (chunk & 1) * 16;
    }
};

typedef shape_t<8, 4, 2, 4, 4> tile256_t;
typedef shape_t<4, 4, 2, 2, 4> tile128_t;

// One operand's copies: the resource that a stage is read from, where it goes on, and what this lane reads of it.
template <class K, lies_t LIES, bool SEG, int OUTER, int COPIES> struct copies_t {
    static constexpr uint32_t BYTES = 2 * OUTER;
    rsrc_t from;
    uint32_t off[COPIES];
    uint32_t full, last, step, beyond; // extents of a whole stage and of one at the contraction's end; beyond: what puts this lane's piece out of bounds there
    int64_t hop[SEG ? 2 : 1];          // from the last stage of a segment to the first of the next

    __device__ __forceinline__ copies_t(const side_t &s, int64_t K_, int64_t at, int64_t begin, uint32_t odd, uint32_t w, uint32_t lane, const int64_t (&starts)[3], int segment)
    {
        const uint32_t pitch = (uint32_t)(s.ld * 2);
        const int64_t most = s.outer - at, first = SEG ? starts[segment] : 0;
        if constexpr (LIES == DOWN) {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const uint32_t row = K::row_of(w * COPIES + i, lane, BYTES);
                off[i] = row * pitch + K::byte_of(row, lane, BYTES);
            }
            const uint32_t wide = (uint32_t)(most * 2 < BYTES ? most * 2 : BYTES); // bytes of a row, in whole words below
            full = ((STAGE - 1) * pitch + wide + 3) & ~3u;
            last = odd ? ((odd - 1) * pitch + wide + 3) & ~3u : 0;
            step = STAGE * pitch;
            beyond = 0;
            from = resource(s.data + first + begin * s.ld + at, full);
        } else {
            const uint32_t piece = (lane & 3) ^ (lane >> 4 & 3); // rows of four lanes: the row's bits 2 and 3 are the lane's 4 and 5
#pragma unroll
            for (int i = 0; i < COPIES; ++i) off[i] = ((w * COPIES + i) * 16 + (lane >> 2)) * pitch + piece * 16;
            const uint32_t rows = (uint32_t)(most < OUTER ? most : OUTER);
            full = (rows - 1) * pitch + 2 * STAGE;
            last = odd ? (rows - 1) * pitch + (odd + 7) / 8 * 16 : 0;
            step = 2 * STAGE;
            beyond = odd && piece * 8 >= odd ? 0x80000000u : 0;
            from = resource(s.data + first + at * s.ld + begin, full);
        }
        if constexpr (SEG) {
            const int64_t run = (K_ / STAGE - 1) * (int64_t)step; // bytes from a segment's first stage to its last
#pragma unroll
            for (int i = 0; i < 2; ++i) hop[i] = (starts[i + 1] - starts[i]) * 2 - run;
        }
    }
    __device__ __forceinline__ void forward(int64_t bytes)
    {
        const uint64_t p = ((uint64_t)from.y << 32 | from.x) + (uint64_t)bytes;
        from.x = (uint32_t)p;
        from.y = (uint32_t)(p >> 32);
    }
};

template <bool F16> __device__ __forceinline__ v4f mfma16(uint4 a, uint4 b, v4f c)
{
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

__device__ __forceinline__ u32x4 lds_read16(uint32_t lds_addr) { return *(const __attribute__((address_space(3))) u32x4 *)lds_addr; }

// acc = the sums over elements begin .. end of the contraction (of all segments, one after the other) of the tile at (n0, d0).  When it returns other waves may
// still read LDS and copies of zeros be on their way: wait_for_copies<0>() and a barrier come before LDS is used for anything else.
template <class K, bool F16, lies_t LA, lies_t LB, bool SEG>
__device__ __forceinline__ void multiply(const product_t &q, int64_t n0, int64_t d0, int64_t begin, int64_t end, uint8_t *smem, v4f (&acc)[K::MT][K::NT])
{
    constexpr int MT = K::MT, NT = K::NT, RING = K::RING;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wn = w / K::WD, wd = w % K::WD;
    const uint32_t base = __builtin_amdgcn_readfirstlane(lds_address(smem));
    int32_t left = (int32_t)(end - begin), ahead = left; // elements from the stage at hand, and from the one that is copied next, on
    int segment = 0;
    uint32_t in = 0, run = 0;
    if constexpr (SEG) {
        run = (uint32_t)(q.K / STAGE);
        segment = (int)(begin / q.K);
        begin -= segment * q.K;
        in = (uint32_t)(begin / STAGE);
    }
    const uint32_t odd = SEG ? 0u : (uint32_t)left % STAGE;
    copies_t<K, LA, SEG, K::TM, K::COPIES_A> a(q.A, q.K, n0, begin, odd, w, lane, q.seg.a, segment);
    copies_t<K, LB, SEG, K::TN, K::COPIES_B> b(q.B, q.K, d0, begin, odd, w, lane, q.seg.b, segment);
    uint32_t to = base, at = base; // slots: copied to next, read next
    const auto after = [&](uint32_t slot) { return slot == base + (RING - 1) * K::SLOT ? base : slot + K::SLOT; };
    uint32_t cut_a = 0, cut_b = 0;
    // The resources of the stage that is copied next: a whole one, the contraction's end, or nothing.  Without a branch: it would end the block that the
    // instructions around are scheduled in.
    const auto trim = [&] {
        a.from.z = ahead >= STAGE ? a.full : ahead > 0 ? a.last : 0;
        b.from.z = ahead >= STAGE ? b.full : ahead > 0 ? b.last : 0;
        if constexpr (LA == ALONG) cut_a = ahead >= STAGE ? 0 : a.beyond;
        if constexpr (LB == ALONG) cut_b = ahead >= STAGE ? 0 : b.beyond;
    };
    const uint32_t own_a = w * K::COPIES_A * 1024, own_b = w * K::COPIES_B * 1024;
    const auto copied = [&] {
        if constexpr (SEG) {
            const bool cross = ++in == run;
            a.forward(cross ? (segment ? a.hop[1] : a.hop[0]) : (int64_t)a.step);
            b.forward(cross ? (segment ? b.hop[1] : b.hop[0]) : (int64_t)b.step);
            in = cross ? 0 : in;
            segment += cross;
        } else {
            a.forward(a.step);
            b.forward(b.step);
        }
        ahead -= STAGE;
        to = after(to);
        trim();
    };
    const auto copy = [&](auto number) {
        constexpr int i = decltype(number)::value;
        if constexpr (i < K::COPIES_A)
            dma16_bounded<i * 1024>(a.from, LA == ALONG ? a.off[i] | cut_a : a.off[i], to + own_a);
        else
            dma16_bounded<K::A + (i - K::COPIES_A) * 1024>(b.from, LB == ALONG ? b.off[i - K::COPIES_A] | cut_b : b.off[i - K::COPIES_A], to + own_b);
    };

    // What this lane reads: the matrix instruction wants the eight elements from 8 (lane / 16) on of row or column lane % 16.  DOWN: four lanes of a group of 16
    // supply the four pieces of a row, of four columns each, and the group receives four rows: two reads.  ALONG: one read.
    const int s16 = lane & 15, g = lane >> 4;
    constexpr int PA = LA == DOWN ? 2 : 1, PB = LB == DOWN ? 2 : 1;
    uint32_t ra[PA == 2 ? MT : 1], rb[PB == 2 ? NT : 1];
    const uint32_t down = 8 * g + (s16 >> 2), along = s16 * 64 + ((g ^ (s16 >> 2)) * 16);
    if constexpr (PA == 2) {
#pragma unroll
        for (int m = 0; m < MT; ++m) ra[m] = down * K::RA + (((wn * MT + m) ^ K::turn_of(down, K::RA)) * 32) + 8 * (s16 & 3);
    } else {
        ra[0] = wn * MT * 1024 + along;
    }
    if constexpr (PB == 2) {
#pragma unroll
        for (int n = 0; n < NT; ++n) rb[n] = K::A + down * K::RB + (((wd * NT + n) ^ K::turn_of(down, K::RB)) * 32) + 8 * (s16 & 3);
    } else {
        rb[0] = K::A + wd * NT * 1024 + along;
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = {};
    u32x2 fa[MT][2], fb[2][NT][2];
    uint32_t lies = 0;
    const auto read_a = [&](int m, int part) {
        if constexpr (PA == 2) {
            if (!part) lies = at + ra[m];
            fa[m][part] = transposed(lies + 4 * part * K::RA);
        } else if (!part) {
            const u32x4 v = lds_read16(at + ra[0] + m * 1024);
            fa[m][0] = v.xy, fa[m][1] = v.zw;
        }
    };
    const auto read_b = [&](int set, int n, int part) {
        if constexpr (PB == 2) {
            if (!part) lies = at + rb[n];
            fb[set][n][part] = transposed(lies + 4 * part * K::RB);
        } else if (!part) {
            const u32x4 v = lds_read16(at + rb[0] + n * 1024);
            fb[set][n][0] = v.xy, fb[set][n][1] = v.zw;
        }
    };
    constexpr int PLACES = MT * NT, BARRIER = NT - 1; // a stage's matrix instructions are places, with what is issued beside each
    constexpr int READS_B = PB * NT, EACH = (READS_B + (MT - 1) * (NT - 2) - 1) / ((MT - 1) * (NT - 2)); // reads of B beside one of the places for them
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
            const uint4 va = make_uint4(fa[m][0].x, fa[m][0].y, fa[m][1].x, fa[m][1].y);
            const uint4 vb = make_uint4(fb[set][n][0].x, fb[set][n][0].y, fb[set][n][1].x, fb[set][n][1].y);
            acc[m][n] = mfma16<F16>(va, vb, acc[m][n]);
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
                    static_for<first, first + EACH < READS_B ? first + EACH : READS_B>([&](auto i) { read_b(set ^ 1, decltype(i)::value / PB, decltype(i)::value % PB); });
            }
            if constexpr (place >= PLACES - K::ISSUED) copy(std::integral_constant<int, place - (PLACES - K::ISSUED)>{});
            ADAHOP_PIN();
        });
        copied();
        left -= STAGE;
    };
    while (left > 0) { // two stages, one of each set of B's registers; the second may be one of zeros
        stage(std::integral_constant<int, 0>{});
        stage(std::integral_constant<int, 1>{});
    }
}

// Which tile a workgroup takes.  Workgroups go round the eight XCDs; each takes a run of tiles, which it walks in columns of four tiles: what runs on it at a time
// shares few tiles of either operand.  SYMMETRIC: only tiles on and below the diagonal, row by row.
template <class K, bool SYMMETRIC> __device__ __forceinline__ void place_of(const product_t &q, int64_t &n0, int64_t &d0)
{
    const uint32_t tiles = SYMMETRIC ? q.nt * (q.nt + 1) / 2 : q.nt * q.dt, id = blockIdx.x, per = tiles / 8, rest = tiles % 8, xcd = id % 8;
    const uint32_t t = xcd * per + (xcd < rest ? xcd : rest) + id / 8;
    if constexpr (SYMMETRIC) {
        uint32_t i = (uint32_t)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while (i * (i + 1) / 2 > t) --i; // the root is to within one
        while ((i + 1) * (i + 2) / 2 <= t) ++i;
        n0 = (int64_t)i * K::TM, d0 = (int64_t)(t - i * (i + 1) / 2) * K::TN;
    } else {
        const uint32_t group = t / (4 * q.dt), in = t - group * 4 * q.dt, high = q.nt - 4 * group < 4 ? q.nt - 4 * group : 4;
        n0 = (int64_t)(4 * group + in % high) * K::TM, d0 = (int64_t)(in / high) * K::TN;
    }
}

// What becomes of the sums is a finish E:
//   COUNTED                        whether rows_of and K_of are looked at
//   E::more_t                      what it reads for four elements
//   more_t get(r, c, have)         that, ahead of its use
//   float4 apply(r, c, have, v, m) finishes C[r, c .. c + have) and stores it; returns the values for put_turned
//   put_turned(c, r, v)            SYMMETRIC: stores eight of them, C[r .. r + 8, c], as row c
struct nothing_t {};

struct store_part_t { // a slice's sums as they are
    typedef nothing_t more_t;
    float *to;
    int64_t ld;
    __device__ __forceinline__ more_t get(int64_t, int64_t, int) const { return {}; }
    __device__ __forceinline__ float4 apply(int64_t r, int64_t c, int have, float4 v, more_t) const
    {
        const float one[4] = {1.0f, 1.0f, 1.0f, 1.0f};
        put4({to, ld, 1}, r, c, have, one, v, make_float4(0.0f, 0.0f, 0.0f, 0.0f));
        return v;
    }
};

// C's rows go by way of a wave's own patch of LDS, 32 at a time, so that a lane has four consecutive columns of a row: 16-byte stores of whole rows.  In
// the accumulators a lane has column lane % 16 of a tile, rows 4 (lane / 16) + i.  What the finish reads is read 32 rows ahead: no load
// passes a store that it might depend on.
template <class K, bool SYMMETRIC, class E>
__device__ __forceinline__ void finish_tile(const product_t &q, int64_t n0, int64_t d0, uint8_t *smem, const v4f (&acc)[K::MT][K::NT], const E &e)
{
    constexpr int MT = K::MT, NT = K::NT, PITCH = 16 * NT + 4, LANES = 4 * NT, STEPS = LANES / 2;
    static_assert(K::WAVES * 32 * PITCH * sizeof(float) <= K::LDS, "the waves' patches fit");
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wn = w / K::WD, wd = w % K::WD;
    const int c4 = lane % LANES * 4, r0 = lane / LANES;
    const int64_t c = d0 + wd * NT * 16 + c4;
    const int have = (int)(q.B.outer - c < 4 ? q.B.outer - c : 4);
    const auto row_at = [&](int m, int i) { return n0 + (wn * MT + m) * 16 + r0 + i * (64 / LANES); };
    float *const patch = reinterpret_cast<float *>(smem) + w * 32 * PITCH;
    typename E::more_t more[2][STEPS];
    const auto get = [&](int m) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (have > 0 && row_at(m, i) < q.A.outer) more[m / 2 & 1][i] = e.get(row_at(m, i), c, have);
    };
    get(0);
    wait_for_copies<0>();
    asm volatile("s_barrier" ::: "memory"); // no wave reads or copies any more
#pragma unroll
    for (int m = 0; m < MT; m += 2) {
        lds_between_lanes();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) patch[(16 * (i >> 2) + 4 * (lane >> 4) + (i & 3)) * PITCH + 16 * n + (lane & 15)] = acc[m + (i >> 2)][n][i & 3];
        lds_between_lanes();
        if (m + 2 < MT) get(m + 2);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            float4 *const v = reinterpret_cast<float4 *>(patch + (r0 + i * (64 / LANES)) * PITCH + c4);
            if (have > 0 && row_at(m, i) < q.A.outer) {
                const float4 done = e.apply(row_at(m, i), c, have, *v, more[m / 2 & 1][i]);
                if constexpr (SYMMETRIC) *v = done;
            }
        }
        if constexpr (SYMMETRIC) {
            if (n0 != d0) { // the tile's mirror image: four lanes have 32 rows of a column
                lds_between_lanes();
                const int64_t r = n0 + (wn * MT + m) * 16 + 8 * (lane & 3);
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const int col = 16 * i + (lane >> 2);
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = patch[(8 * (lane & 3) + j) * PITCH + col];
                    if (d0 + wd * NT * 16 + col < q.B.outer && r < q.A.outer) e.put_turned(d0 + wd * NT * 16 + col, r, v);
                }
            }
        }
    }
}

// SYMMETRIC: A = B up to segments, so is C; both outer extents are one multiple of 32.
template <class K, bool F16, lies_t LA, lies_t LB, bool SEG, bool SYMMETRIC, class E> __global__ __launch_bounds__(K::THREADS, 2) void k_product16(product_t q, E e)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    int64_t n0, d0;
    place_of<K, SYMMETRIC>(q, n0, d0);
    float *const part = q.part + (int64_t)blockIdx.y * q.A.outer * q.B.outer;
    int64_t all = SEG ? q.K * q.seg.count : q.K;
    if constexpr (E::COUNTED) {
        if (q.K_of) all = __builtin_amdgcn_readfirstlane(*q.K_of);
        if (q.rows_of) {
            q.A.outer = __builtin_amdgcn_readfirstlane(*q.rows_of);
            if (n0 >= q.A.outer) return;
        }
    }
    const int64_t begin = (int64_t)blockIdx.y * q.slice, till = begin + q.slice < all ? begin + q.slice : all, end = till < begin ? begin : till;
    v4f acc[K::MT][K::NT];
    multiply<K, F16, LA, LB, SEG>(q, n0, d0, begin, end, smem, acc);
    if (q.part)
        finish_tile<K, false>(q, n0, d0, smem, acc, store_part_t{part, q.B.outer});
    else
        finish_tile<K, SYMMETRIC>(q, n0, d0, smem, acc, e);
}

// The sums of the slices, in their order, finished.  A lane has four columns.  SYMMETRIC: `tile` is the tiles' edge; above the diagonal of tiles the sums are those of the
// mirror image.
template <bool SYMMETRIC, class E>
__global__ __launch_bounds__(256) void k_join16(const float *part, int slices, int64_t rows, int64_t cols, int tile, const int32_t *rows_of, E e)
{
    const int64_t c = ((int64_t)blockIdx.y * 64 + (threadIdx.x & 63)) * 4, r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (c >= cols || r >= (rows_of ? *rows_of : rows)) return;
    const int have = (int)(cols - c < 4 ? cols - c : 4);
    const typename E::more_t more = e.get(r, c, have);
    float v[4] = {};
    const bool turned = SYMMETRIC && r / tile < c / tile;
    const float *p = turned ? part + c * cols + r : part + r * cols + c;
    const int64_t across = turned ? cols : 1;
    if (have == 4 && !turned) {
#pragma unroll 4
        for (int s = 0; s < slices; ++s, p += rows * cols) {
            const u32x4 a = *reinterpret_cast<const u32x4_e4 *>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += __uint_as_float(a[i]);
        }
    } else {
        for (int s = 0; s < slices; ++s, p += rows * cols)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < have) v[i] += p[i * across];
    }
    e.apply(r, c, have, make_float4(v[0], v[1], v[2], v[3]), more);
}

// to = factor v + add, of bf16 or float.  place (or nullptr): which of `to`'s rows row r is.  by (or nullptr): a number on the device that the factor is multiplied by.
struct grad_t {
    static constexpr bool COUNTED = true;
    typedef float4 more_t;
    adahop_tensor_t to, add;
    const int32_t *place;
    float factor;
    const float *by;
    __device__ __forceinline__ more_t get(int64_t r, int64_t c, int have) const { return get4(add, r, c, have); }
    __device__ __forceinline__ float4 apply(int64_t r, int64_t c, int have, float4 v, more_t more) const
    {
        const float f = by ? factor * *by : factor, scale[4] = {f, f, f, f};
        put4(to, place ? place[r] : r, c, have, scale, v, more);
        return v;
    }
};

// ---- host ----------------------------------------------------------------------------------------------------------------------
// Tiles and slices of a product by its expected time.
struct plan16_t {
    bool large;
    int slices;
    int64_t slice;
    size_t part_bytes;
};

// As measured for the weight gradient from a checkpoint (plan_of in wgrad8.hip), in microseconds on 256 compute units: a stage of a round of workgroups 0.7 with the large
// tiles, one workgroup per compute unit; with the small ones 0.5 where there are two per compute unit, 0.3 where there is one; a round's beginning and end 4 and 2.5.
inline plan16_t plan16(int64_t rows, int64_t cols, int64_t K, bool symmetric)
{
    const auto count = [&](int64_t t) { return symmetric ? ceil_div(rows, t) * (ceil_div(rows, t) + 1) / 2 : ceil_div(rows, t) * ceil_div(cols, t); };
    const int64_t stages = ceil_div(K, STAGE), large = count(256), small = count(128);
    plan16_t p = {};
    double best = 0.0;
    for (int64_t slices = 1; slices <= 64 && (slices == 1 || stages / slices >= 8); ++slices) {
        const int64_t each = ceil_div(ceil_div(stages, slices), 2) * 2; // stages per slice; the kernel takes them in pairs
        const int64_t number = ceil_div(stages, each);
        const double join = number > 1 ? 6.0 + (double)number * rows * cols * 8 / 5e6 : 0.0;
        const int64_t rounds = small * number / 512, over = small * number % 512;
        const double in_large = ceil_div(large * number, 256) * (4.0 + 0.7 * each) + join;
        const double in_small = (rounds + (over > 0)) * 2.5 + (rounds * 0.5 + (over > 256 ? 0.5 : over > 0 ? 0.3 : 0.0)) * each + join;
        const double t = in_large < in_small ? in_large : in_small;
        if (p.slices == 0 || t < best) {
            best = t;
            p.large = in_large < in_small;
            p.slices = (int)number;
            p.slice = each * STAGE;
        }
        if (join > best) break;
    }
    p.part_bytes = p.slices > 1 ? (size_t)p.slices * rows * cols * sizeof(float) : 0;
    return p;
}

template <class K, bool F16, lies_t LA, lies_t LB, bool SEG, bool SYMMETRIC, class E> inline int configure_product16()
{
    return check_hip(hipFuncSetAttribute(reinterpret_cast<const void *>(&k_product16<K, F16, LA, LB, SEG, SYMMETRIC, E>), hipFuncAttributeMaxDynamicSharedMemorySize, K::LDS));
}

template <class K, bool F16, lies_t LA, lies_t LB, bool SEG, bool SYMMETRIC, class E> inline int launch_tiles16(product_t &q, int slices, const E &e, hipStream_t st)
{
    q.nt = (uint32_t)ceil_div(q.A.outer, K::TM), q.dt = (uint32_t)ceil_div(q.B.outer, K::TN);
    k_product16<K, F16, LA, LB, SEG, SYMMETRIC, E><<<dim3(SYMMETRIC ? q.nt * (q.nt + 1) / 2 : q.nt * q.dt, slices), K::THREADS, K::LDS, st>>>(q, e);
    return check_launch();
}

// A product as planned.  part: room for plan.part_bytes.
template <bool F16, lies_t LA, lies_t LB, bool SEG, bool SYMMETRIC, class E>
inline int launch_product16(const plan16_t &plan, product_t q, const E &e, void *part, hipStream_t st)
{
    q.slice = plan.slice;
    q.part = plan.slices > 1 ? static_cast<float *>(part) : nullptr;
    const int rc = plan.large ? launch_tiles16<tile256_t, F16, LA, LB, SEG, SYMMETRIC>(q, plan.slices, e, st)
                              : launch_tiles16<tile128_t, F16, LA, LB, SEG, SYMMETRIC>(q, plan.slices, e, st);
    if (rc != ADAHOP_OK || !q.part) return rc;
    k_join16<SYMMETRIC, E><<<dim3((unsigned)ceil_div(q.A.outer, 4), (unsigned)ceil_div(q.B.outer, 256)), 256, 0, st>>>(q.part, plan.slices, q.A.outer, q.B.outer,
                                                                                                                 plan.large ? 256 : 128, q.rows_of, e);
    return check_launch();
}

template <bool F16, lies_t LA, lies_t LB, bool SEG, bool SYMMETRIC, class E> inline int configure_both16()
{
    const int rc = configure_product16<tile256_t, F16, LA, LB, SEG, SYMMETRIC, E>();
    return rc == ADAHOP_OK ? configure_product16<tile128_t, F16, LA, LB, SEG, SYMMETRIC, E>() : rc;
}

} // namespace

} // namespace adahop

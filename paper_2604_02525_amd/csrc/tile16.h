// Products of 16-bit operands (bf16 or fp16) on the matrix cores with sums in fp32, for the operators at the end of a training step:
//
//     C[r, c] = sum_k A(r, k) B(c, k)
//
// Either operand may hold the contraction along its rows (ALONG, [outer][K]) or down its columns (DOWN, [K][outer]), so that no operand is ever transposed
// in memory: a gradient of logits [tokens][vocabulary] enters one product by its rows and another by its columns.
//
// What bounds it: the matrix cores, on large problems their power (16384 x 8192 x 65536, three such products: 1.37 PFLOP/s, the library's bf16 product of 8192 x 8192 x 8192 1.33 with contiguous
// contraction, 1.04 with both operands strided); where a compute unit has one workgroup of 128 x 128, LDS: half a slab
// takes 0.23 us, its matrix instructions 0.11, 48 KB read from LDS and 16 KB copied there 0.21 at 128 bytes a cycle (four waves would read 32 KB, but there is nothing to hide a wave's waits behind then: 413 us
// for an update that takes 359).
//
// The scheme is that of the weight gradient from a checkpoint (wgrad8.hip): both operands go to LDS by copies that pass no register, a wave's 16 x 16 x 32 instructions are fed
// from LDS 32 elements of the contraction ahead.  A DOWN operand is turned by the transposing reads of LDS; an ALONG one is read as it lies, 16 bytes (eight elements
// of a row) per lane.  What lies outside an operand reads as zero, in both.  Here LDS holds slabs of 64 elements of the contraction rather than stages of 32: an ALONG
// operand's rows are then fetched in whole lines of 128 bytes (where both are DOWN, whose rows are long, in halves all the same, further ahead).  In halves of them the L2s' requests, not the matrix cores, set the pace: 32 compute units' took as long as their matrix instructions
// (matrix cores busy 53 % against 79 % with both operands DOWN).
//
// LDS layout of a slab of an ALONG operand: 128 bytes a row, its eight pieces of 16 bytes exchanged by a number for the row's bits 1 to 3 (exchange_of).  A read of 16 bytes per lane serves
// sixteen lanes at a time, not lanes in a row: any two of the sixteen are in different banks for sixteen rows with one piece, for four rows at either end with one piece and
// the eight between them with its neighbour, and for eight rows with two neighbouring pieces.  With a number that does so for the first alone half of the reads' cycles were conflicts (counted).
// What conflicts are left are at the ends of symmetric products: put_mirror and k_direct16 read eight rows of a patch in neighbouring lanes eight rows apart, a multiple of 32 banks (33 to 40 % of the LDS cycles of
// a product of few slabs, 4 % of a long one's).
#pragma once
#include "tile_copies.h"

namespace adahop {

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

enum lies_t { ALONG, DOWN };

constexpr int SLAB = 64; // of the contraction: two matrix instructions'

__device__ __forceinline__ uint32_t exchange_of(uint32_t q) { return (2 * q & 7) ^ (q >> 2) * 5; } // 0, 2, 4, 6, 5, 7, 1, 3

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
    int64_t K;       // a multiple of 8 where an operand is ALONG; of 64 with several segments
    uint32_t nt, dt; // tiles along A's outer index and B's
    // The first `whole` tiles are a workgroup's each.  Of the others a workgroup has one of `slices` slices of the contraction (`slice` elements of all segments' K, a
    // multiple of 64), whose sums go to part, [tile][slice][TM][TN]; with one slice they are whole too.
    uint32_t whole, slices;
    int64_t slice;
    float *part;
    segments_t seg;
    const int32_t *rows_of, *K_of; // (or nullptr) how many of A's outer indices and of the contraction's elements there are, where only the device knows
};

// Tiles of C by WN x WD waves of 16 MT x 16 NT, a ring of RING slabs.
template <int MT_, int NT_, int WN_, int WD_, int RING_> struct shape_t {
    static constexpr int MT = MT_, NT = NT_, WN = WN_, WD = WD_, RING = RING_;
    static constexpr int WAVES = WN * WD, THREADS = 64 * WAVES, TM = 16 * WN * MT, TN = 16 * WD * NT, RA = 2 * TM, RB = 2 * TN; // bytes of a row of a DOWN slab
    static constexpr uint32_t A = SLAB * RA, B = SLAB * RB, SLOT = A + B, LDS = RING * SLOT;
    static constexpr int COPIES = A / 1024 / (WAVES / 2); // per wave and slab: half of the waves copy A, the others B
    static_assert(TM == TN && COPIES * (WAVES / 2) * 1024 == A && COPIES % 2 == 0, "whole copies");
    // DOWN: by what the pieces of 32 bytes of a row are exchanged, so that the eight rows of a transposing read of half a wave (four consecutive ones and those 8 further on)
    // lie in different banks.  Rows of a multiple of 256 bytes begin at the same bank: by bits 0, 1 and 3 of the row.  Rows of 128 or 384: two of them lie apart, by bits 1 and 3.
    static __device__ __forceinline__ uint32_t turn_of(uint32_t row, uint32_t bytes) { return bytes % 256 ? (row >> 1 & 1) | (row >> 2 & 2) : (row & 3) | (row >> 1 & 4); }
    // What lane l of copy number `copy` of a slab reads: its row, and the byte in it
    static __device__ __forceinline__ uint32_t row_of(uint32_t copy, uint32_t l, uint32_t bytes) { return (copy * 1024 + l * 16) / bytes; }
    static __device__ __forceinline__ uint32_t byte_of(uint32_t row, uint32_t l, uint32_t copy, uint32_t bytes)
    {
        const uint32_t chunk = (copy * 1024 + l * 16 - row * bytes) / 16;
        return ((chunk >> 1) ^ turn_of(row, bytes)) * 32 + (chunk & 1) * 16;
    }
};

typedef shape_t<8, 4, 2, 4, 2> tile256_t;
typedef shape_t<6, 3, 2, 4, 3> tile192_t;
typedef shape_t<4, 4, 2, 2, 2> tile128_t;       // two workgroups on a compute unit
typedef shape_t<2, 4, 4, 2, 4> tile128_alone_t; // one: a slab takes less time than its copies, so they go further ahead.  2048 x 2048 updated: 359 us, with tile128_t 459, with a
                                                // ring of four and four waves 413; two of these tiles on a compute unit (rings of two) were slower or the same

// A wave's copies, all of one operand: the resource that a slab is read from, where it goes on, and what this lane reads of it.
// UNIT: elements of the contraction that are copied at a time, a slab or half of one.
template <class K, bool SEG, int UNIT> struct copies_t {
    static constexpr int OUTER = K::TM, COPIES = K::COPIES * UNIT / SLAB;
    static constexpr uint32_t BYTES = 2 * OUTER;
    rsrc_t from;
    uint32_t off[COPIES];
    uint32_t full, last, step, beyond[2]; // extents of a whole unit and of one at the contraction's end; beyond: what puts this lane's piece of copies of either parity out of bounds there
    int64_t hop[SEG ? 2 : 1];             // from the last unit of a segment to the first of the next

    // w: which of the waves that copy this operand
    __device__ __forceinline__ void set(lies_t lies, const side_t &s, int64_t K_, int64_t at, int64_t begin, uint32_t odd, uint32_t w, uint32_t lane, const int64_t (&starts)[3], int segment)
    {
        const uint32_t pitch = (uint32_t)(s.ld * 2);
        const int64_t most = s.outer - at, first = SEG ? starts[segment] : 0;
        if (lies == DOWN) {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const uint32_t row = K::row_of(w * COPIES + i, lane, BYTES);
                off[i] = row * pitch + K::byte_of(row, lane, w * COPIES + i, BYTES);
            }
            const uint32_t wide = (uint32_t)(most * 2 < BYTES ? most * 2 : BYTES); // bytes of a row, in whole words below
            full = ((UNIT - 1) * pitch + wide + 3) & ~3u;
            last = odd ? ((odd - 1) * pitch + wide + 3) & ~3u : 0;
            step = UNIT * pitch;
            beyond[0] = beyond[1] = 0;
            from = resource(s.data + first + begin * s.ld + at, full);
        } else {
            // eight lanes have a row: its bits 1 and 2 are the lane's 4 and 5, bit 3 is the copy's parity
            const uint32_t piece[2] = {(lane & 7) ^ exchange_of(lane >> 4), (lane & 7) ^ exchange_of(4 + (lane >> 4))};
#pragma unroll
            for (int i = 0; i < COPIES; ++i) off[i] = ((w * COPIES + i) * 8 + (lane >> 3)) * pitch + piece[i & 1] * 16;
            const uint32_t rows = (uint32_t)(most < OUTER ? most : OUTER);
            full = (rows - 1) * pitch + 2 * SLAB;
            last = odd ? (rows - 1) * pitch + (odd + 7) / 8 * 16 : 0;
            step = 2 * SLAB;
#pragma unroll
            for (int i = 0; i < 2; ++i) beyond[i] = odd && piece[i] * 8 >= odd ? 0x80000000u : 0;
            from = resource(s.data + first + at * s.ld + begin, full);
        }
        if constexpr (SEG) {
            const int64_t run = (K_ / UNIT - 1) * (int64_t)step; // bytes from a segment's first unit to its last
#pragma unroll
            for (int i = 0; i < 2; ++i) hop[i] = (starts[i + 1] - starts[i]) * 2 - run;
        }
    }
    // Into scalar registers, which the copies take the resource from: it is the same in all lanes, but the compiler may have come to it another way.
    static __device__ __forceinline__ uint32_t one(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane(v); }
    __device__ __forceinline__ void settle_from() { from.x = one(from.x), from.y = one(from.y), from.z = one(from.z), from.w = one(from.w); }
    __device__ __forceinline__ void settle()
    {
        settle_from();
        full = one(full), last = one(last), step = one(step);
        if constexpr (SEG) {
#pragma unroll
            for (int i = 0; i < 2; ++i) hop[i] = (int64_t)((uint64_t)one((uint32_t)((uint64_t)hop[i] >> 32)) << 32 | one((uint32_t)hop[i]));
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
    constexpr bool FINE = LA == DOWN && LB == DOWN; // halves of slabs are copied, 2 RING - 1 ahead
    constexpr int UNIT = FINE ? SLAB / 2 : SLAB;
    typedef copies_t<K, SEG, UNIT> mine_t;
    constexpr int COPIES = mine_t::COPIES;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), wn = w / K::WD, wd = w % K::WD;
    const uint32_t base = __builtin_amdgcn_readfirstlane(lds_address(smem));
    int32_t left = __builtin_amdgcn_readfirstlane((int32_t)(end - begin)), ahead = left; // elements from the slab at hand, and from what is copied next, on
    int segment = 0;
    uint32_t in = 0, run = 0;
    if constexpr (SEG) {
        run = (uint32_t)(q.K / UNIT);
        segment = __builtin_amdgcn_readfirstlane((int)(begin / q.K));
        begin -= segment * q.K;
        in = __builtin_amdgcn_readfirstlane((uint32_t)(begin / UNIT));
    }
    const uint32_t odd = SEG ? 0u : (uint32_t)left % UNIT;
    mine_t mine;
    const bool of_b = w >= K::WAVES / 2;
    if (of_b)
        mine.set(LB, q.B, q.K, d0, begin, odd, w - K::WAVES / 2, lane, q.seg.b, segment);
    else
        mine.set(LA, q.A, q.K, n0, begin, odd, w, lane, q.seg.a, segment);
    mine.settle();
    const uint32_t own = of_b ? K::A + (w - K::WAVES / 2) * COPIES * 1024 : w * COPIES * 1024;
    uint32_t to = base, at = base; // the slabs that are copied to next and read next
    const auto after = [&](uint32_t slot) { return slot == base + (RING - 1) * K::SLOT ? base : slot + K::SLOT; };
    uint32_t cut[2] = {};
    // The resource of what is copied next: a whole unit, the contraction's end, or nothing.  Without a branch: it would end the block that the
    // instructions around are scheduled in.
    const auto trim = [&] {
        mine.from.z = ahead >= UNIT ? mine.full : ahead > 0 ? mine.last : 0;
        mine.settle_from();
        if constexpr (LA == ALONG || LB == ALONG) cut[0] = ahead >= UNIT ? 0 : mine.beyond[0], cut[1] = ahead >= UNIT ? 0 : mine.beyond[1];
    };
    const auto copied = [&](bool whole_slab) { // whole_slab: with this unit it is
        if constexpr (SEG) {
            const bool cross = ++in == run;
            mine.forward(cross ? (segment ? mine.hop[1] : mine.hop[0]) : (int64_t)mine.step);
            in = cross ? 0 : in;
            segment += cross;
        } else {
            mine.forward(mine.step);
        }
        ahead -= UNIT;
        to = whole_slab ? after(to) : to;
        trim();
    };
    const auto copy = [&](auto number, auto half) {
        constexpr int i = decltype(number)::value;
        constexpr uint32_t lies_at = decltype(half)::value * (SLAB / 2) * K::RA + i * 1024; // half: which of a slab's a FINE unit is
        dma16_bounded<lies_at>(mine.from, LA == ALONG || LB == ALONG ? mine.off[i] | cut[i & 1] : mine.off[i], __builtin_amdgcn_readfirstlane(to + own));
    };

    // What this lane reads of a half slab: the matrix instruction wants the eight elements from 8 (lane / 16) on of row or column lane % 16.  DOWN: four lanes of a group of
    // 16 supply the four pieces of a row, of four columns each, and the group receives four rows: two reads.  ALONG: one read.
    const int s16 = lane & 15, g = lane >> 4;
    constexpr int PA = LA == DOWN ? 2 : 1, PB = LB == DOWN ? 2 : 1;
    uint32_t ra[PA == 2 ? MT : 2], rb[PB == 2 ? NT : 2]; // ALONG: of either half
    const uint32_t down = 8 * g + (s16 >> 2), along = s16 * 128 + ((g ^ exchange_of(s16 >> 1)) * 16);
    if constexpr (PA == 2) {
#pragma unroll
        for (int m = 0; m < MT; ++m) ra[m] = down * K::RA + (((wn * MT + m) ^ K::turn_of(down, K::RA)) * 32) + 8 * (s16 & 3);
    } else {
        ra[0] = wn * MT * 2048 + along, ra[1] = wn * MT * 2048 + (along ^ 64);
    }
    if constexpr (PB == 2) {
#pragma unroll
        for (int n = 0; n < NT; ++n) rb[n] = K::A + down * K::RB + (((wd * NT + n) ^ K::turn_of(down, K::RB)) * 32) + 8 * (s16 & 3);
    } else {
        rb[0] = K::A + wd * NT * 2048 + along, rb[1] = K::A + wd * NT * 2048 + (along ^ 64);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[m][n] = {};
    u32x2 fa[MT][2], fb[2][NT][2];
    uint32_t lies = 0;
    const auto read_a = [&](int half, int m, int part) {
        if constexpr (PA == 2) {
            if (!part) lies = at + ra[m];
            fa[m][part] = transposed(lies + (32 * half + 4 * part) * K::RA);
        } else if (!part) {
            const u32x4 v = lds_read16(at + ra[half] + m * 2048);
            fa[m][0] = v.xy, fa[m][1] = v.zw;
        }
    };
    const auto read_b = [&](int half, int n, int part) { // into the set of registers of that half
        if constexpr (PB == 2) {
            if (!part) lies = at + rb[n];
            fb[half][n][part] = transposed(lies + (32 * half + 4 * part) * K::RB);
        } else if (!part) {
            const u32x4 v = lds_read16(at + rb[half] + n * 2048);
            fb[half][n][0] = v.xy, fb[half][n][1] = v.zw;
        }
    };
    constexpr int PLACES = MT * NT, BARRIER = NT - 1; // a half slab's matrix instructions are places, with what is issued beside each
    constexpr int READS_B = PB * NT, EACH = (READS_B + (MT - 1) * (NT - 2) - 1) / ((MT - 1) * (NT - 2)); // reads of B beside one of the places for them
    constexpr int APART = !FINE && (PLACES - NT) / COPIES > 2 ? 2 : 1, FIRST = FINE ? PLACES - COPIES : BARRIER + 1; // places from one copy to the next, the first one's
    static_assert(NT > 2 && COPIES * APART <= PLACES - NT, "what goes beside the matrix instructions fits");

    trim();
    static_for<0, FINE ? 2 * RING - 1 : RING>([&](auto unit) {
        constexpr int half = FINE ? decltype(unit)::value & 1 : 0;
        static_for<0, COPIES>([&](auto i) { copy(i, std::integral_constant<int, half>{}); });
        copied(!FINE || half);
    });
    wait_for_copies<(FINE ? 2 * RING - 2 : RING - 1) * COPIES>();
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
        read_a(0, m, 0), read_a(0, m, 1);
    }
    ADAHOP_PIN();
    // A's operands are read again, for the next half, behind the last of the NT matrix instructions that use them, B's into the other set of registers.  The last of a unit is
    // read behind its last half's first instructions; after the barrier that follows, what comes RING slabs later goes in its place, and the next unit, copied
    // for at least the time of one and a half halves with two slabs, is there for all waves.
    const auto half = [&](auto which) {
        constexpr int now = decltype(which)::value, next = now ^ 1;
        static_for<0, PLACES>([&](auto number) {
            constexpr int place = decltype(number)::value, m = place / NT, n = place % NT;
            const uint4 va = make_uint4(fa[m][0].x, fa[m][0].y, fa[m][1].x, fa[m][1].y);
            const uint4 vb = make_uint4(fb[now][n][0].x, fb[now][n][0].y, fb[now][n][1].x, fb[now][n][1].y);
            acc[m][n] = mfma16<F16>(va, vb, acc[m][n]);
            if constexpr (m == 0 && n < 2) read_a(now, MT - 1, n);
            if constexpr ((FINE || now == 1) && place == BARRIER) {
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((FINE ? 2 * RING - 3 : RING - 2) * COPIES) : "memory");
                if constexpr (now == 1) at = after(at);
            }
            if constexpr (m > 0) {
                constexpr int first = ((m - 1) * (NT - 2) + n - 2) * EACH;
                if constexpr (n < 2)
                    read_a(next, m - 1, n);
                else
                    static_for<first, first + EACH < READS_B ? first + EACH : READS_B>([&](auto i) { read_b(next, decltype(i)::value / PB, decltype(i)::value % PB); });
            }
            if constexpr ((FINE || now == 1) && place >= FIRST && (place - FIRST) % APART == 0 && (place - FIRST) / APART < COPIES)
                copy(std::integral_constant<int, (place - FIRST) / APART>{}, std::integral_constant<int, FINE ? next : 0>{});
            ADAHOP_PIN();
        });
        if constexpr (FINE || now == 1) copied(!FINE || now == 0); // (FINE: in a first half the second one of a slab, in a second half the next one's first)
    };
    while (left > 0) {
        half(std::integral_constant<int, 0>{});
        half(std::integral_constant<int, 1>{});
        left -= SLAB;
    }
}

// Where tile t is.  A run of tiles goes by columns of four: what an XCD works on at a time shares few tiles of either operand.  SYMMETRIC: only
// tiles on and below the diagonal.
template <class K, bool SYMMETRIC> __device__ __forceinline__ void place_of(uint32_t nt, uint32_t dt, uint32_t t, int64_t &n0, int64_t &d0)
{
    if constexpr (SYMMETRIC) { // groups of four rows: 16 g + 10 tiles in group g, its columns up to 4 g + 1 whole
        uint32_t g = (uint32_t)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.125f);
        while (g && 8 * g * g + 2 * g > t) --g; // the root is to within one
        while (8 * (g + 1) * (g + 1) + 2 * (g + 1) <= t) ++g;
        const uint32_t in = t - (8 * g * g + 2 * g), high = nt - 4 * g < 4 ? nt - 4 * g : 4, even = high * (4 * g + 1);
        uint32_t i = in % high, j = in / high;
        if (in >= even) { // the last columns' ends: high - 1 tiles, high - 2, ...
            uint32_t left = in - even, down = 1;
            for (; left >= high - down; ++down) left -= high - down;
            i = down + left, j = 4 * g + down;
        }
        n0 = (int64_t)(4 * g + i) * K::TM, d0 = (int64_t)j * K::TN;
    } else {
        const uint32_t group = t / (4 * dt), in = t - group * 4 * dt, high = nt - 4 * group < 4 ? nt - 4 * group : 4;
        n0 = (int64_t)(4 * group + in % high) * K::TM, d0 = (int64_t)(in / high) * K::TN;
    }
}

// Workgroups go round the eight XCDs; each takes a run of `tiles` tiles.
__device__ __forceinline__ uint32_t run_of_xcd(uint32_t id, uint32_t tiles)
{
    const uint32_t per = tiles / 8, rest = tiles % 8, xcd = id % 8;
    return xcd * per + (xcd < rest ? xcd : rest) + id / 8;
}

// Where a lane's four elements are: a row and a column for the whole wave, and the lane's from there on.
struct spot_t {
    int64_t r0, c0;
    uint32_t r, c;
    __device__ __forceinline__ int64_t row() const { return r0 + r; }
    __device__ __forceinline__ int64_t col() const { return c0 + c; }
    // its element of an array of rows of ld < 2^26 elements: a wave's address in scalar registers, 32 bits of the lane's own
    template <class T> __device__ __forceinline__ T *in(T *base, int64_t ld) const
    {
        typedef typename std::conditional<std::is_const<T>::value, const char, char>::type byte_t;
        return reinterpret_cast<T *>(reinterpret_cast<byte_t *>(base + r0 * ld + c0) + (uint32_t)((r * (uint32_t)ld + c) * sizeof(T)));
    }
};

// Four elements of a tensor of rows of ld < 2^26, and storing them: get4 and put4 with a wave's address in scalar registers.
__device__ __forceinline__ float4 get4_at(const adahop_tensor_t &t, const spot_t &s, int have)
{
    float o[4] = {};
    if (t.f32) {
        const uint32_t *const p = s.in(static_cast<const uint32_t *>(t.data), t.ld);
        if (have == 4) {
            const u32x4 a = *reinterpret_cast<const u32x4_e4 *>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(a[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < have) o[i] = __uint_as_float(p[i]);
        }
    } else {
        const uint16_t *const p = s.in(static_cast<const uint16_t *>(t.data), t.ld);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) o[i] = bf16_one(p[i]);
    }
    return make_float4(o[0], o[1], o[2], o[3]);
}

__device__ __forceinline__ void put4_at(const adahop_tensor_t &t, const spot_t &s, int have, const float (&v)[4])
{
    if (t.f32) {
        uint32_t *const p = s.in(static_cast<uint32_t *>(t.data), t.ld);
        if (have == 4) {
            *reinterpret_cast<u32x4_e4 *>(p) = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < have) p[i] = __float_as_uint(v[i]);
        }
    } else {
        typedef uint32_t u32x2_e2 __attribute__((ext_vector_type(2), aligned(2), may_alias));
        uint16_t *const p = s.in(static_cast<uint16_t *>(t.data), t.ld);
        const u32x2 w = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
        if (have == 4) {
            *reinterpret_cast<u32x2_e2 *>(p) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < have) p[i] = (uint16_t)(w[i >> 1] >> 16 * (i & 1));
        }
    }
}

// What becomes of the sums is a finish E:
//   COUNTED                        whether rows_of and K_of are looked at
//   E::column_t, column(c, have)   what it reads for four columns, once for all their rows
//   E::more_t, get(spot, have)     what it reads for four elements, ahead of its use (by AHEAD - 1 blocks of 32 rows)
//   float4 apply(spot, have, v, column, more) finishes and stores the first `have` of them; returns the values for put_turned
//   put_turned(c, r, v)            SYMMETRIC: stores eight of them, C[r .. r + 8, c], as row c
struct nothing_t {};


struct store_part_t { // a slice's sums as they are
    static constexpr int AHEAD = 2;
    typedef nothing_t column_t, more_t;
    float *to; // of the tile at (n0, d0)
    int64_t n0, d0, ld;
    __device__ __forceinline__ column_t column(int64_t, int) const { return {}; }
    __device__ __forceinline__ more_t get(const spot_t &, int) const { return {}; }
    __device__ __forceinline__ float4 apply(const spot_t &s, int, float4 v, column_t, more_t) const
    {
        *reinterpret_cast<float4 *>(spot_t{s.r0 - n0, s.c0 - d0, s.r, s.c}.in(to, ld)) = v;
        return v;
    }
};

// The mirror image of a wave's patch of 32 rows of 16 NT columns at (r0, c0): four lanes have the 32 rows of a column.
template <int NT, class E> __device__ __forceinline__ void put_mirror(const product_t &q, int64_t r0, int64_t c0, const float *patch, const E &e)
{
    constexpr int PITCH = 16 * NT + 4;
    const int lane = threadIdx.x & 63, down = 8 * (lane & 3);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int col = 16 * i + (lane >> 2);
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = patch[(down + j) * PITCH + col];
        if (c0 + col < q.B.outer && r0 + down < q.A.outer) e.put_turned(c0 + col, r0 + down, v);
    }
}

// C's rows go by way of a wave's own patch of LDS, 32 at a time, so that a lane has four consecutive columns of a row: 16-byte stores of whole rows.  In
// the accumulators a lane has column lane % 16 of a tile, rows 4 (lane / 16) + i.  What the finish reads is read a block of rows ahead (AHEAD = 2), or with the block itself (1): no load
// passes a store that it might depend on.  Two blocks ahead measured the same.
template <class K, bool SYMMETRIC, class E>
__device__ __forceinline__ void finish_tile(const product_t &q, int64_t n0, int64_t d0, uint8_t *smem, const v4f (&acc)[K::MT][K::NT], const E &e)
{
    constexpr int MT = K::MT, NT = K::NT, PITCH = 16 * NT + 4, LANES = 4 * NT, ROWS = 64 / LANES, STEPS = (32 + ROWS - 1) / ROWS, AHEAD = E::AHEAD; // lanes of a row, rows at a time
    static_assert(K::WAVES * 32 * PITCH * sizeof(float) <= K::LDS, "the waves' patches fit");
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wn = w / K::WD, wd = w % K::WD;
    const int c4 = lane % LANES * 4, r0 = lane / LANES;
    const int64_t c0 = d0 + wd * NT * 16, c = c0 + c4, first = n0 + wn * MT * 16;
    const int have = (int)(q.B.outer - c < 4 ? q.B.outer - c : 4);
    // whether step i of the rows from 16 m on is one of this lane's
    const auto is = [&](int m, int i) { return have > 0 && r0 < q.A.outer - first - m * 16 - i * ROWS && (32 % ROWS == 0 || (r0 < ROWS && r0 + i * ROWS < 32)); };
    const auto spot = [&](int m, int i) { return spot_t{first + m * 16 + i * ROWS, c0, (uint32_t)r0, (uint32_t)c4}; };
    float *const patch = reinterpret_cast<float *>(smem) + w * 32 * PITCH;
    typename E::column_t column;
    if (have > 0) column = e.column(c, have);
    typename E::more_t more[AHEAD][STEPS];
    const auto get = [&](int m) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
            if (is(m, i)) more[m / 2 % AHEAD][i] = e.get(spot(m, i), have);
    };
    wait_for_copies<0>(); // those of zeros behind the last stage
#pragma unroll
    for (int m = 0; m < 2 * (AHEAD - 1) && m < MT; m += 2) get(m);
    asm volatile("s_barrier" ::: "memory"); // no wave reads or copies any more
#pragma unroll
    for (int m = 0; m < MT; m += 2) {
        lds_between_lanes();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) patch[(16 * (i >> 2) + 4 * (lane >> 4) + (i & 3)) * PITCH + 16 * n + (lane & 15)] = acc[m + (i >> 2)][n][i & 3];
        lds_between_lanes();
        if (m + 2 * (AHEAD - 1) < MT) get(m + 2 * (AHEAD - 1));
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            float4 *const v = reinterpret_cast<float4 *>(patch + (r0 + i * ROWS) * PITCH + c4);
            if (is(m, i)) {
                const float4 done = e.apply(spot(m, i), have, *v, column, more[m / 2 % AHEAD][i]);
                if constexpr (SYMMETRIC) *v = done;
            }
        }
        if constexpr (SYMMETRIC) {
            if (n0 != d0) {
                lds_between_lanes();
                put_mirror<NT>(q, first + m * 16, c0, patch, e);
            }
        }
    }
}

// SYMMETRIC: A = B up to segments, so is C; both outer extents are one multiple of 64.
template <class K, bool F16, lies_t LA, lies_t LB, bool SEG, bool SYMMETRIC, class E> __global__ __launch_bounds__(K::THREADS, 2) void k_product16(product_t q, E e)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    int64_t n0, d0, begin = 0, all = SEG ? q.K * q.seg.count : q.K, end = all;
    const uint32_t past = blockIdx.x - q.whole;
    const bool sliced = blockIdx.x >= q.whole && q.slices > 1;
    place_of<K, SYMMETRIC>(q.nt, q.dt, blockIdx.x < q.whole ? run_of_xcd(blockIdx.x, q.whole) : q.whole + past / q.slices, n0, d0);
    if constexpr (E::COUNTED) {
        if (q.K_of) end = all = __builtin_amdgcn_readfirstlane(*q.K_of);
        if (q.rows_of) {
            q.A.outer = __builtin_amdgcn_readfirstlane(*q.rows_of);
            if (n0 >= q.A.outer) return;
        }
    }
    if (sliced) {
        begin = past % q.slices * q.slice;
        end = begin + q.slice < all ? begin + q.slice : all < begin ? begin : all;
    }
    v4f acc[K::MT][K::NT];
    multiply<K, F16, LA, LB, SEG>(q, n0, d0, begin, end, smem, acc);
    if (sliced)
        finish_tile<K, false>(q, n0, d0, smem, acc, store_part_t{q.part + (int64_t)past * K::TM * K::TN, n0, d0, K::TN});
    else
        finish_tile<K, SYMMETRIC>(q, n0, d0, smem, acc, e);
}

// The sums of the slices of the tiles that have some, finished: a workgroup has 32 rows of 32 columns of a tile, each of its waves every fourth slice, and the waves' sums are added in
// their order.  (One wave for all slices: 31 of them of three tiles took 23 us.)
// TURNED: the values go to put_turned, too, where the tile is not on a SYMMETRIC product's diagonal.
template <class K, bool SYMMETRIC, bool TURNED, class E> __global__ __launch_bounds__(256) void k_join16(product_t q, E e)
{
    constexpr int PITCH = 36, ACROSS = K::TN / 32, PATCHES = K::TM / 32 * ACROSS;
    __shared__ __attribute__((aligned(16))) float sums[4][32 * PITCH];
    const uint32_t tail = blockIdx.x / PATCHES, in = blockIdx.x % PATCHES;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c4 = (lane & 7) * 4, r0 = lane >> 3;
    int64_t n0, d0;
    place_of<K, SYMMETRIC>(q.nt, q.dt, q.whole + tail, n0, d0);
    if constexpr (E::COUNTED) {
        if (q.rows_of) q.A.outer = *q.rows_of;
    }
    const int64_t first = n0 + in / ACROSS * 32, c0 = d0 + in % ACROSS * 32, c = c0 + c4;
    const spot_t spot = {first + 8 * w, c0, (uint32_t)r0, (uint32_t)c4};
    const int have = (int)(q.B.outer - c < 4 ? q.B.outer - c : 4);
    const bool is = have > 0 && spot.row() < q.A.outer;
    typename E::column_t column;
    typename E::more_t more;
    if (is) column = e.column(c, have), more = e.get(spot, have);
    // of every element of a tile, whether C has it or not
    const float *p = q.part + ((int64_t)tail * q.slices + w) * K::TM * K::TN + (first - n0 + r0) * K::TN + (c - d0);
    float4 sum[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (uint32_t s = w; s < q.slices; s += 4, p += 4 * K::TM * K::TN)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 v = *reinterpret_cast<const float4 *>(p + i * 8 * K::TN);
            sum[i] = make_float4(sum[i].x + v.x, sum[i].y + v.y, sum[i].z + v.z, sum[i].w + v.w);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float4 *>(sums[w] + (r0 + 8 * i) * PITCH + c4) = sum[i];
    __syncthreads();
    float *const at = sums[0] + (r0 + 8 * w) * PITCH + c4;
    if (is) {
        float4 v = *reinterpret_cast<const float4 *>(at);
#pragma unroll
        for (int k = 1; k < 4; ++k) {
            const float4 o = *reinterpret_cast<const float4 *>(at + k * 32 * PITCH);
            v = make_float4(v.x + o.x, v.y + o.y, v.z + o.z, v.w + o.w);
        }
        v = e.apply(spot, have, v, column, more);
        if constexpr (TURNED) *reinterpret_cast<float4 *>(at) = v;
    }
    if constexpr (TURNED) {
        __syncthreads();
        if (w || (SYMMETRIC && n0 == d0)) return;
        put_mirror<2>(q, first, c0, sums[0], e);
    }
}

// to = factor v + add, of bf16 or float.  place (or nullptr): which of `to`'s rows row r is.  by (or nullptr): a number on the device that the factor is multiplied by, of
// tokens of which there are *tokens: without one it takes no part, whatever it is.
struct grad_t {
    static constexpr bool COUNTED = true;
    static constexpr int AHEAD = 2;
    typedef float column_t; // the factor
    struct more_t {
        float4 add;
        int32_t place;
    };
    adahop_tensor_t to, add;
    const int32_t *place;
    float factor;
    const float *by;
    const int32_t *tokens;
    __device__ __forceinline__ column_t column(int64_t, int) const { return by && *tokens ? factor * *by : factor; }
    __device__ __forceinline__ more_t get(const spot_t &s, int have) const { return {get4(add, s.row(), s.col(), have), place ? place[s.row()] : 0}; }
    __device__ __forceinline__ float4 apply(const spot_t &s, int have, float4 v, column_t f, const more_t &m) const
    {
        const float scale[4] = {f, f, f, f};
        put4(to, place ? m.place : s.row(), s.col(), have, scale, v, m.add);
        return v;
    }
};

// ---- small products -----------------------------------------------------------------------------------------------------------------
// Both operands ALONG, all extents multiples of 64: tiles of 64 x 64, whose four waves share the contraction.  A wave copies what it needs itself, two slabs ahead, to LDS of
// its own: nothing waits for a barrier before the waves' sums meet.  What the finish reads is read before the first slab.  Where tiles are few, latency is all that
// counts.  136 tiles of a symmetric product with a contraction of 1024: 18.5 us with tiles of 128, and 11.6 us with operands loaded straight to registers (a quarter of a wave reads 16 rows
// then, each lane's 16 bytes an access of their own).
struct direct_t {
    static constexpr int TM = 64, TN = 64, WAVES = 4, THREADS = 256, PITCH = 68;
    static constexpr uint32_t SIDE = 64 * 2 * SLAB, STEP = 2 * SIDE, OWN = 2 * STEP, LDS = WAVES * OWN;
    static_assert(WAVES * 64 * PITCH * sizeof(float) <= LDS, "the waves' sums fit");
};

// TURNED: the finish's values go to put_turned, too, where the tile is not on a SYMMETRIC product's diagonal.
template <bool F16, bool SEG, bool SYMMETRIC, bool TURNED, class E> __global__ __launch_bounds__(direct_t::THREADS) void k_direct16(product_t q, E e)
{
    typedef direct_t K;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    float *const sums = reinterpret_cast<float *>(smem); // [wave][64][PITCH]
    int64_t n0, d0;
    const uint32_t past = blockIdx.x - q.whole;
    const bool sliced = blockIdx.x >= q.whole && q.slices > 1;
    place_of<K, SYMMETRIC>(q.nt, q.dt, blockIdx.x < q.whole ? run_of_xcd(blockIdx.x, q.whole) : q.whole + past / q.slices, n0, d0);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), s16 = lane & 15, g = lane >> 4;
    // the contraction's slabs: this slice's, and this wave's of them
    const int all = (int)((SEG ? q.K * q.seg.count : q.K) / SLAB), of_slice = sliced ? (int)(q.slice / SLAB) : all;
    const int from = sliced ? (int)(past % q.slices) * of_slice : 0, till = from + of_slice < all ? from + of_slice : all;
    const int first = __builtin_amdgcn_readfirstlane(from + (till - from) * w / K::WAVES), steps = __builtin_amdgcn_readfirstlane(from + (till - from) * (w + 1) / K::WAVES) - first;
    const auto spot = [&](int p) { return spot_t{n0 + 16 * p + 4 * w, d0, (uint32_t)g, (uint32_t)s16 * 4}; };
    typename E::column_t column;
    typename E::more_t more[4];
    if (!sliced) {
        column = e.column(spot(0).col(), 4);
#pragma unroll
        for (int p = 0; p < 4; ++p) more[p] = e.get(spot(p), 4);
    }
    // eight lanes have a row of a copy of eight; the row's bits 1 and 2 are the lane's 4 and 5, bit 3 is the copy's parity
    const uint32_t mine = lds_address(smem) + w * K::OWN;
    uint32_t off_a[2], off_b[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t piece = (lane & 7) ^ exchange_of(4 * i + (lane >> 4));
        off_a[i] = ((uint32_t)(lane >> 3) * (uint32_t)q.A.ld + 8 * piece) * 2, off_b[i] = ((uint32_t)(lane >> 3) * (uint32_t)q.B.ld + 8 * piece) * 2;
    }
    const uint16_t *const pa = q.A.data + n0 * q.A.ld, *const pb = q.B.data + d0 * q.B.ld;
    const int run = (int)(q.K / SLAB);
    const auto copy = [&](int step, int half) {
        int64_t a = 0, b = 0;
        step += first;
        if constexpr (SEG) {
            const int segment = step >= run ? step >= 2 * run ? 2 : 1 : 0;
            a = segment == 2 ? q.seg.a[2] : segment ? q.seg.a[1] : q.seg.a[0];
            b = segment == 2 ? q.seg.b[2] : segment ? q.seg.b[1] : q.seg.b[0];
            step -= segment * run;
        }
        const uint8_t *const ca = reinterpret_cast<const uint8_t *>(pa + a + step * SLAB), *const cb = reinterpret_cast<const uint8_t *>(pb + b + step * SLAB);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dma16(ca + i * 16 * q.A.ld, off_a[i & 1], mine + half * K::STEP + i * 1024);
            dma16(cb + i * 16 * q.B.ld, off_b[i & 1], mine + half * K::STEP + K::SIDE + i * 1024);
        }
    };
    v4f acc[4][4];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[m][n] = {};
    const uint32_t along = mine + s16 * 128 + (g ^ exchange_of(s16 >> 1)) * 16;
    if (steps > 0) copy(0, 0);
    if (steps > 1) copy(1, 1);
    for (int i = 0; i < steps; ++i) {
        if (i + 1 < steps)
            wait_for_copies<16>();
        else
            wait_for_copies<0>();
        u32x4 fa[2][4], fb[2][4];
        const uint32_t at = along + (i & 1) * K::STEP;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int m = 0; m < 4; ++m) fa[h][m] = lds_read16((at ^ 64 * h) + m * 2048), fb[h][m] = lds_read16((at ^ 64 * h) + K::SIDE + m * 2048);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); // read: what follows may go in its place
        if (i + 2 < steps) copy(i + 2, i & 1);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int n = 0; n < 4; ++n) acc[m][n] = mfma16<F16>(__builtin_bit_cast(uint4, fa[h][m]), __builtin_bit_cast(uint4, fb[h][n]), acc[m][n]);
    }
    __syncthreads();
    float *const own = sums + w * 64 * K::PITCH;
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) own[(16 * m + 4 * g + i) * K::PITCH + 16 * n + s16] = acc[m][n][i];
    __syncthreads();
    float4 v[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        v[p] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < K::WAVES; ++k) {
            const float4 o = *reinterpret_cast<const float4 *>(sums + (k * 64 + 16 * p + 4 * w + g) * K::PITCH + s16 * 4);
            v[p] = make_float4(v[p].x + o.x, v[p].y + o.y, v[p].z + o.z, v[p].w + o.w);
        }
    }
    if (sliced) {
        const store_part_t part = {q.part + (int64_t)past * K::TM * K::TN, n0, d0, K::TN};
#pragma unroll
        for (int p = 0; p < 4; ++p) part.apply(spot(p), 4, v[p], {}, {});
        return;
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) v[p] = e.apply(spot(p), 4, v[p], column, more[p]);
    if constexpr (TURNED) {
        if (SYMMETRIC && n0 == d0) return;
        __syncthreads();
#pragma unroll
        for (int p = 0; p < 4; ++p) *reinterpret_cast<float4 *>(sums + (16 * p + 4 * w + g) * K::PITCH + s16 * 4) = v[p];
        __syncthreads();
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int col = (threadIdx.x >> 3) + 32 * p, down = 8 * (threadIdx.x & 7);
            float t[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = sums[(down + j) * K::PITCH + col];
            e.put_turned(d0 + col, n0 + down, t);
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------------------
// Tiles and slices of a product by its expected time.
struct plan16_t {
    int edge;
    uint32_t tiles, whole, slices; // of the tiles behind the whole ones
    int64_t slice;
    size_t part_bytes;
    double time; // microseconds, as expected
};

// In microseconds, on 256 compute units: half a slab of a round of workgroups takes 0.74 with tiles of 256, 0.43 of 192, one workgroup per compute unit; of 128 0.6 where there are two
// per compute unit, 0.23 where there is one; a round's beginning and end 12, 10 and 6.  Whole rounds of tiles are computed whole.  What is left is cut into slices if they,
// their sums' way to memory and back and one launch more take less time than another round.  `slices_at_most` = 1: never.  `small`: tiles of 128 alone.
constexpr double ROUND192 = 0.43, ALONE128 = 0.23;

inline plan16_t plan16(int64_t rows, int64_t cols, int64_t K, bool symmetric, int64_t slices_at_most = 64, bool small = false)
{
    plan16_t best = {};
    const int64_t stages = ceil_div(K, SLAB) * 2; // of 32 elements of the contraction
    for (const int edge : {256, 192, 128}) {
        if (small && edge > 128) continue;
        const int64_t room = edge > 128 ? 256 : 512, down = ceil_div(rows, edge), across = ceil_div(cols, edge);
        const int64_t tiles = symmetric ? down * (down + 1) / 2 : down * across, rest = tiles % room;
        const double each = edge == 256 ? 0.74 : edge == 192 ? ROUND192 : 0.6, ends = edge == 256 ? 12.0 : edge == 192 ? 10.0 : 6.0, whole = (double)(tiles / room) * (ends + each * (double)stages);
        const auto a_round = [&](int64_t workgroups, int64_t of) { return ends + (workgroups <= 256 && edge == 128 ? ALONE128 : each) * (double)of; };
        plan16_t p = {edge, (uint32_t)tiles, (uint32_t)tiles, 1, 0, 0, 0.0};
        double time = whole + (rest ? a_round(rest, stages) : 0.0);
        for (int64_t s = 2; rest && s <= slices_at_most && stages / s >= 4; ++s) {
            const int64_t of = ceil_div(ceil_div(stages, s), 2) * 2, number = ceil_div(stages, of);
            const double t = whole + (double)(rest * number / room) * (ends + each * (double)of) + (rest * number % room ? a_round(rest * number % room, of) : 0.0) + 8.0 +
                             (double)(rest * number * edge * edge) * 8 / 5e6;
            if (t < time) {
                time = t;
                p.whole = (uint32_t)(tiles - rest), p.slices = (uint32_t)number, p.slice = of * 32;
                p.part_bytes = (size_t)rest * number * edge * edge * sizeof(float);
            }
        }
        if (!best.edge || time < best.time) best = p, best.time = time;
    }
    return best;
}

// The same for k_direct16: a round of 256 tiles takes DIRECT_ENDS, and DIRECT_STEP for each 32 of the contraction; slices as above.
constexpr double DIRECT_ENDS = 4.0, DIRECT_STEP = 0.14;

inline plan16_t plan_direct16(int64_t rows, int64_t cols, int64_t K, bool symmetric)
{
    const int64_t down = ceil_div(rows, 64), tiles = symmetric ? down * (down + 1) / 2 : down * ceil_div(cols, 64), steps = ceil_div(K, SLAB) * 2;
    plan16_t best = {64, (uint32_t)tiles, (uint32_t)tiles, 1, 0, 0, (double)ceil_div(tiles, 256) * (DIRECT_ENDS + DIRECT_STEP * (double)steps)};
    for (int64_t s = 2; s <= 32 && steps / s >= 16 && tiles * s <= 512; ++s) {
        const int64_t of = ceil_div(ceil_div(steps, s), 2) * 2, number = ceil_div(steps, of);
        const double time = (double)ceil_div(tiles * number, 256) * (DIRECT_ENDS + DIRECT_STEP * (double)of) + 5.0;
        if (time < best.time) best = {64, (uint32_t)tiles, 0, (uint32_t)number, of * 32, (size_t)tiles * number * 64 * 64 * sizeof(float), time};
    }
    return best;
}

// Whether a plan's tiles of 128 have a compute unit each.
inline bool alone16(const plan16_t &plan) { return plan.edge == 128 && plan.whole + (plan.tiles - plan.whole) * plan.slices <= 256; }

template <class K, bool F16, lies_t LA, lies_t LB, bool SEG, bool SYMMETRIC, class E> inline int configure_product16()
{
    return check_hip(hipFuncSetAttribute(reinterpret_cast<const void *>(&k_product16<K, F16, LA, LB, SEG, SYMMETRIC, E>), hipFuncAttributeMaxDynamicSharedMemorySize, K::LDS));
}

template <class K, bool F16, lies_t LA, lies_t LB, bool SEG, bool SYMMETRIC, class E> inline int launch_tiles16(product_t &q, const plan16_t &plan, const E &e, hipStream_t st)
{
    const uint32_t rest = plan.tiles - plan.whole;
    q.nt = (uint32_t)ceil_div(q.A.outer, K::TM), q.dt = (uint32_t)ceil_div(q.B.outer, K::TN);
    k_product16<K, F16, LA, LB, SEG, SYMMETRIC, E><<<plan.whole + rest * plan.slices, K::THREADS, K::LDS, st>>>(q, e);
    const int rc = check_launch();
    if (rc != ADAHOP_OK || !rest) return rc;
    k_join16<K, SYMMETRIC, SYMMETRIC, E><<<rest * (K::TM / 32) * (K::TN / 32), 256, 0, st>>>(q, e);
    return check_launch();
}

// A product as planned (SEG: with `small`).  part: room for plan.part_bytes.
template <bool F16, lies_t LA, lies_t LB, bool SEG, bool SYMMETRIC, class E>
inline int launch_product16(const plan16_t &plan, product_t q, const E &e, void *part, hipStream_t st)
{
    q.whole = plan.whole, q.slices = plan.slices, q.slice = plan.slice;
    q.part = static_cast<float *>(part);
    if constexpr (!SEG) {
        if (plan.edge == 256) return launch_tiles16<tile256_t, F16, LA, LB, SEG, SYMMETRIC>(q, plan, e, st);
        if (plan.edge == 192) return launch_tiles16<tile192_t, F16, LA, LB, SEG, SYMMETRIC>(q, plan, e, st);
    }
    return alone16(plan) ? launch_tiles16<tile128_alone_t, F16, LA, LB, SEG, SYMMETRIC>(q, plan, e, st) : launch_tiles16<tile128_t, F16, LA, LB, SEG, SYMMETRIC>(q, plan, e, st);
}

template <bool F16, bool SEG, bool SYMMETRIC, bool TURNED, class E> inline int configure_direct16()
{
    return check_hip(hipFuncSetAttribute(reinterpret_cast<const void *>(&k_direct16<F16, SEG, SYMMETRIC, TURNED, E>), hipFuncAttributeMaxDynamicSharedMemorySize, direct_t::LDS));
}

template <bool F16, bool SEG, bool SYMMETRIC, bool TURNED, class E> inline int launch_direct16(const plan16_t &plan, product_t q, const E &e, void *part, hipStream_t st)
{
    typedef direct_t K;
    const uint32_t rest = plan.tiles - plan.whole;
    q.whole = plan.whole, q.slices = plan.slices, q.slice = plan.slice;
    q.part = static_cast<float *>(part);
    q.nt = (uint32_t)(q.A.outer / 64), q.dt = (uint32_t)(q.B.outer / 64);
    k_direct16<F16, SEG, SYMMETRIC, TURNED, E><<<plan.whole + rest * plan.slices, K::THREADS, K::LDS, st>>>(q, e);
    const int rc = check_launch();
    if (rc != ADAHOP_OK || !rest) return rc;
    k_join16<K, SYMMETRIC, TURNED, E><<<rest * 4, 256, 0, st>>>(q, e);
    return check_launch();
}

template <bool F16, lies_t LA, lies_t LB, bool SEG, bool SYMMETRIC, class E> inline int configure_all16()
{
    int rc = ADAHOP_OK;
    if constexpr (!SEG) {
        rc = configure_product16<tile256_t, F16, LA, LB, SEG, SYMMETRIC, E>();
        if (rc == ADAHOP_OK) rc = configure_product16<tile192_t, F16, LA, LB, SEG, SYMMETRIC, E>();
    }
    if (rc == ADAHOP_OK) rc = configure_product16<tile128_alone_t, F16, LA, LB, SEG, SYMMETRIC, E>();
    return rc == ADAHOP_OK ? configure_product16<tile128_t, F16, LA, LB, SEG, SYMMETRIC, E>() : rc;
}

} // namespace

} // namespace adahop

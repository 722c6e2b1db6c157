// Softmax cross entropy over a vocabulary, from the last hidden states and the output weights, without the logits in memory:
//
//     z[t, v] = logit_scale sum_d h[t, d] w[v, d],   lse[t] = log sum_v exp z[t, v],   loss[t] = lse - z[t, y_t] + z_loss lse^2
//     dz[t, v] = d_loss[t] logit_scale ((1 + 2 z_loss lse) exp(z - lse) - [v = y_t]),   d_h = dz w,   d_w = dz^T h
//
// Backward, the tokens that have a target are gathered first: the others take no part in either gradient, whatever they hold.  What they save: d_w's contraction is
// of the tokens that are left; the logits and d_h have fewer tiles, but not less time until few are left, as those that remain are the first XCDs' (8192 x 4096 x 32000 with one d_loss, none, half, nine tenths of the tokens
// without a target: 4.91, 4.02 and 2.99 ms).  The forward pass computes all of them: lse is that of every token.
//
// Forward: a tile of z (words of the vocabulary by tokens) stays in the matrix cores' accumulators and leaves two numbers per token, its largest logit and
// the sum of exponentials relative to that; a second kernel joins the tiles of a token.  Backward: a piece of the vocabulary at a time, z is
// computed again, dz of the piece goes to the workspace in bf16 and enters both gradients' products.
//
// The rounding of dz to bf16 (each element by at most 2^-8 of itself) is what the matrix cores take; it is of the size of the gradients' own rounding and, as
// errors of the elements are independent, adds less than that to a sum over them.  Where all tokens have one d_loss (that of a mean), it and logit_scale are left out of
// dz and multiply the products' fp32 sums: the target's element, mostly the largest of its row, is then -1 and little more, which loses next to nothing (8192 x 4096 x 32000: d_h 2.6e-3
// of its norm off with them inside).  All sums, lse and the loss are fp32.
//
// What bounds it: the matrix cores' power (8192 x 4096 x 32000: forward 1.60 to 1.67 ms on different cards, 1.29 to 1.35 PFLOP/s; backward, three such products, 4.87 to 5.01 ms, 1.29 to 1.32; 16384 x 8192 x 65536 backward 38.7 to
// 39.8 ms, 1.33 to 1.36);
// a few tokens: reading w (one of 4096 against 32000 words: 45 us, 5.8 TB/s).  Forward that writes no logits spares 2 T V bytes twice, 0.2 ms of the 1.6 at the copy's rate.
#include <math.h>

#include "row_sums.h"
#include "tile16.h"

namespace adahop {

namespace {

struct loss_t {
    const int64_t *targets;
    int64_t T, V;
    float logit_scale, z_loss;
};

// ---- forward --------------------------------------------------------------------------------------------------------------------
struct stats_t {
    loss_t p;
    int64_t v0, tile, tiles; // the launch's first word, and its first of the parts of the vocabulary that a token has numbers of
    float2 *part;            // [T][tiles]: largest logit, sum of exponentials relative to it
    float *at;               // [T]: the target's logit
};

// A largest logit and the sum of exponentials relative to it, of two sets of words.
__device__ __forceinline__ float2 joined(float2 a, float2 b)
{
    const float top = fmaxf(a.x, b.x), from = top == -INFINITY ? 0.0f : top;
    return make_float2(top, a.y * __expf(a.x - from) + b.y * __expf(b.x - from));
}

template <int MASK> __device__ __forceinline__ float across(float v) { return __shfl_xor(v, MASK); }

// A: w (rows of a tile: words), B: h (columns: tokens).  A lane has one token per 16 columns and a quarter of the tile's words of its wave: most of a token's
// maximum and sum are formed in its registers.
template <class K> __global__ __launch_bounds__(K::THREADS, 2) void k_ce_stats(product_t q, stats_t e)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    int64_t n0, d0;
    place_of<K, false>(q.nt, q.dt, run_of_xcd(blockIdx.x, q.nt * q.dt), n0, d0);
    v4f acc[K::MT][K::NT];
    multiply<K, false, ALONG, ALONG, false>(q, n0, d0, 0, q.K, smem, acc);
    wait_for_copies<0>();
    __syncthreads();
    float2 *const of_wave = reinterpret_cast<float2 *>(smem); // [WN][TN]
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, wn = w / K::WD, wd = w % K::WD;
    const int first = (int)(q.A.outer - n0 < K::TM ? q.A.outer - n0 : K::TM) - wn * K::MT * 16 - 4 * (lane >> 4); // words of this lane's from its first on, below its rows' count
#pragma unroll
    for (int n = 0; n < K::NT; ++n) {
        const int64_t t = d0 + (wd * K::NT + n) * 16 + (lane & 15);
        const int64_t y = t < q.B.outer ? e.p.targets[t] - e.v0 - n0 - wn * K::MT * 16 - 4 * (lane >> 4) : -1;
        const int mine = y >= 0 && y < K::MT * 16 && y < first ? (int)y : -1; // the target as a row of this lane's, if it is one
        float top = -INFINITY, sum = 0.0f, at = 0.0f;
        bool is = false;
#pragma unroll
        for (int m = 0; m < K::MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float z = acc[m][n][i] * e.p.logit_scale;
                acc[m][n][i] = m * 16 + i < first ? z : -INFINITY;
                top = fmaxf(top, acc[m][n][i]);
                at = mine == m * 16 + i ? z : at;
                is |= mine == m * 16 + i;
            }
        top = fmaxf(top, across<16>(top));
        top = fmaxf(top, across<32>(top));
        const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int m = 0; m < K::MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += __expf(acc[m][n][i] - from);
        sum += across<16>(sum);
        sum += across<32>(sum);
        if (is) e.at[t] = at;
        if (lane < 16) of_wave[wn * K::TN + (wd * K::NT + n) * 16 + lane] = make_float2(top, sum);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < K::TN; i += K::THREADS) {
        if (d0 + i >= q.B.outer) break;
        float2 s = of_wave[i];
#pragma unroll
        for (int k = 1; k < K::WN; ++k) s = joined(s, of_wave[k * K::TN + i]);
        e.part[(d0 + i) * e.tiles + e.tile + n0 / K::TM] = s;
    }
}

// Up to FEW tokens (the likelihood of what has just been generated): bound by reading w once, a tile of tokens would be almost empty.  A wave forms the logits of four words
// at a time, 512 elements of their rows a step, h from LDS; it keeps a token's largest logit and sum of exponentials over its words.
constexpr int FEW = 8;

template <int T> __global__ __launch_bounds__(256, 2) void k_ce_few(side_t w, side_t h, int64_t K, stats_t e)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    uint16_t *const own = reinterpret_cast<uint16_t *>(smem); // [T][pitch]
    const int lane = threadIdx.x & 63;
    const int64_t pitch = (K + 511) / 512 * 512;
    for (int64_t i = threadIdx.x * 8; i < T * pitch; i += 256 * 8) {
        const int64_t t = i / pitch, k = i - t * pitch;
        *reinterpret_cast<u32x4 *>(own + i) = t < h.outer && k < K ? *reinterpret_cast<const u32x4 *>(h.data + t * h.ld + k) : u32x4{0, 0, 0, 0};
    }
    __syncthreads();
    const int64_t waves = (int64_t)gridDim.x * 4, wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    float top[T], sum[T];
#pragma unroll
    for (int t = 0; t < T; ++t) top[t] = -INFINITY, sum[t] = 0.0f;
    for (int64_t v0 = wave * 4; v0 < w.outer; v0 += waves * 4) {
        const uint16_t *row[4]; // (those behind the vocabulary: its last word's)
#pragma unroll
        for (int r = 0; r < 4; ++r) row[r] = w.data + (v0 + r < w.outer ? v0 + r : w.outer - 1) * w.ld;
        float acc[4][T] = {};
        u32x4 next[4];
        const auto load = [&](int64_t k) {
#pragma unroll
            for (int r = 0; r < 4; ++r) next[r] = k + lane * 8 < K ? __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(row[r] + k + lane * 8)) : u32x4{0, 0, 0, 0};
        };
        load(0);
        for (int64_t k = 0; k < pitch; k += 512) {
            float x[4][8];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[r][i] = i & 1 ? bf16_hi(next[r][i >> 1]) : bf16_lo(next[r][i >> 1]);
            if (k + 512 < pitch) load(k + 512);
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const u32x4 y = *reinterpret_cast<const u32x4 *>(own + t * pitch + k + lane * 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float b = i & 1 ? bf16_hi(y[i >> 1]) : bf16_lo(y[i >> 1]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[r][t] = fmaf(x[r][i], b, acc[r][t]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < T; ++t) {
            if (t >= h.outer) break;
            const int64_t y = e.p.targets[t] - v0;
            float z[4], most = top[t];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                z[r] = sum64(acc[r][t]) * e.p.logit_scale;
                if (y == r && lane == 0 && v0 + r < w.outer) e.at[t] = z[r];
                if (v0 + r >= w.outer) z[r] = -INFINITY;
                most = fmaxf(most, z[r]);
            }
            const float from = most == -INFINITY ? 0.0f : most;
            sum[t] *= __expf(top[t] - from);
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[t] += __expf(z[r] - from);
            top[t] = most;
        }
    }
    __syncthreads();
    float2 *const of_wave = reinterpret_cast<float2 *>(smem); // [4][T]
    if (lane == 0)
#pragma unroll
        for (int t = 0; t < T; ++t) of_wave[(threadIdx.x >> 6) * T + t] = make_float2(top[t], sum[t]);
    __syncthreads();
    const int t = threadIdx.x;
    if (t >= h.outer) return;
    float2 s = of_wave[t];
#pragma unroll
    for (int k = 1; k < 4; ++k) s = joined(s, of_wave[k * T + t]);
    e.part[t * gridDim.x + blockIdx.x] = s;
}

// One wave per token: its tiles' numbers joined, the loss.
__global__ __launch_bounds__(256) void k_ce_join(loss_t p, const float2 *part, const float *at, int tiles, float *loss, float *lse)
{
    const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (t >= p.T) return;
    float2 all = make_float2(-INFINITY, 0.0f);
#pragma unroll 4
    for (int i = lane; i < tiles; i += 64) all = joined(all, part[t * tiles + i]);
    const float top = all.x;
    float sum = all.y;
    float most = top;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) most = fmaxf(most, __shfl_xor(most, k));
    const float from = most == -INFINITY ? 0.0f : most;
    sum = sum64(sum * __expf(top - from));
    if (lane) return;
    const float l = from + logf(sum);
    const int64_t y = p.targets[t];
    if (lse) lse[t] = l;
    if (loss) loss[t] = y < 0 ? 0.0f : y < p.V ? l - at[t] + p.z_loss * l * l : NAN;
}

// ---- backward -------------------------------------------------------------------------------------------------------------------
// What dz of a token that has a target needs of it.
struct alignas(16) token_t { // (read in one load)
    float lse, gain; // gain: what exp(z - lse) - [v = target] is multiplied by
    int32_t target;
};

// dz of a piece of the vocabulary from its logits (rows: tokens, columns: words from v0 on), rounded to bf16; zeros from the piece's end to the row's.
struct dlogits_t {
    static constexpr bool COUNTED = true;
    static constexpr int AHEAD = 2;
    typedef nothing_t column_t;
    typedef token_t more_t;
    const token_t *rows;
    float logit_scale, z_loss;
    int64_t v0, words, ld;
    uint16_t *dz;
    __device__ __forceinline__ column_t column(int64_t, int) const { return {}; }
    __device__ __forceinline__ more_t get(const spot_t &at, int) const { return rows[at.row()]; }
    __device__ __forceinline__ float4 apply(const spot_t &at, int have, float4 v, column_t, const more_t &m) const
    {
        const int64_t c = at.col();
        const float z[4] = {v.x, v.y, v.z, v.w}, s = 1.0f + 2.0f * z_loss * m.lse;
        const int64_t hit = m.target - v0 - c;
        float d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            d[i] = (s * __expf(z[i] * logit_scale - m.lse) - (hit == i ? 1.0f : 0.0f)) * m.gain;
            if (i >= have) d[i] = 0.0f;
        }
        uint16_t *const to = at.in(dz, ld); // 8-byte aligned
        *reinterpret_cast<u32x2 *>(to) = u32x2{bf16_pair(d[0], d[1]), bf16_pair(d[2], d[3])};
        if (c + 4 >= words && c + 4 < ld) *reinterpret_cast<u32x2 *>(to + 4) = u32x2{0, 0}; // rows are whole pieces of eight
        return v;
    }
};

// An operand of rows that a copy to LDS cannot take as they are, laid out anew: rows of whole pieces of eight, zeros behind their end.
__global__ __launch_bounds__(256) void k_lay_out(adahop_tensor_t x, int64_t rows, int64_t cols, uint16_t *out, int64_t ld)
{
    const int64_t pieces = ld / 8, all = rows * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces, c = (i - r * pieces) * 8;
        const raw8<false> v = load8<false>(x.data, r * x.ld + c, (int)(cols - c < 8 ? cols - c : 8));
        *reinterpret_cast<u32x4 *>(out + r * ld + c) = v.w[0];
    }
}

// Which tokens have a target, in their order, and how many: one workgroup, 8192 tokens at a time.
__global__ __launch_bounds__(1024) void k_ce_tokens(const int64_t *targets, int64_t T, int32_t *token, int32_t *count)
{
    constexpr int EACH = 8;
    __shared__ int of_wave[16];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int before = 0; // found so far
    for (int64_t from = 0; from < T; from += 1024 * EACH) {
        const int64_t t = from + threadIdx.x * EACH;
        uint32_t has = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) has |= (uint32_t)(t + i < T && targets[t + i] >= 0) << i;
        const int mine = __popc(has);
        int sum = mine; // of this lane and those before it
#pragma unroll
        for (int k = 1; k < 64; k *= 2) {
            const int o = __shfl_up(sum, k);
            sum += lane >= k ? o : 0;
        }
        if (lane == 63) of_wave[w] = sum;
        __syncthreads();
        int at = before + sum - mine, all = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            at += i < w ? of_wave[i] : 0;
            all += of_wave[i];
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (has >> i & 1) token[at++] = (int32_t)(t + i);
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) *count = before;
}

// h's rows of these tokens, one after the other, and what dz needs of them.  A workgroup has a row; those past the last token's have nothing to do.
// factor: logit_scale, or 1 where it and a d_loss for all tokens come later (then d_loss = nullptr).
__global__ __launch_bounds__(256) void k_gather(adahop_tensor_t x, int64_t cols, loss_t p, const float *lse, const float *d_loss, int64_t d_loss_stride, float factor, const int32_t *token,
                                                const int32_t *count, uint16_t *out, int64_t ld, token_t *rows)
{
    const int64_t r = blockIdx.x;
    if (r >= *count) return;
    const int32_t t = token[r];
    if (threadIdx.x == 0) {
        const int64_t y = p.targets[t];
        const float g = (d_loss ? d_loss[t * d_loss_stride] : 1.0f) * factor;
        rows[r] = {lse[t], y < p.V ? g : NAN, (int32_t)(y < p.V ? y : 0)};
    }
    const int64_t from = t * x.ld;
    for (int64_t c = threadIdx.x * 8; c < ld; c += 256 * 8) {
        const raw8<false> v = load8<false>(x.data, from + c, (int)(cols - c < 8 ? cols - c : 8));
        *reinterpret_cast<u32x4 *>(out + r * ld + c) = v.w[0];
    }
}

// d_h of the tokens without a target.
__global__ __launch_bounds__(256) void k_ce_zeros(const int64_t *targets, int64_t cols, adahop_tensor_t out)
{
    const int64_t t = blockIdx.x;
    if (targets[t] >= 0) return;
    const float zero[8] = {};
    for (int64_t c = threadIdx.x * 8; c < cols; c += 256 * 8) store8_any(out, t * out.ld + c, (int)(cols - c < 8 ? cols - c : 8), zero);
}

// d_w of up to FEW_D_W tokens: bound by writing it.  A lane has four features of all tokens in registers and forms their sums for eight words at a time, in the tokens' order; what dz
// it needs is the same for a whole workgroup and comes by scalar loads.  131072 words of 2048 features, bf16: 152 us, as a product's tiles, which would be nothing but their beginnings and ends,
// 229 (and by matrix instructions of 32 tokens without tiles 178 to 192); twice the tokens take 328 for 65536 words of 4096, and the tiles 212.
constexpr int FEW_D_W = 8, D_W_WORDS = 32; // words of a workgroup

__global__ __launch_bounds__(256) void k_ce_d_w_few(const uint16_t *__restrict__ h, int64_t ldh, const uint16_t *__restrict__ dz, int64_t ld, const int32_t *__restrict__ count, int64_t words,
                                                    int64_t cols, grad_t e)
{
    const int n = *count;
    const int64_t c = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4, v0 = (int64_t)blockIdx.x * D_W_WORDS;
    if (c >= cols) return;
    const int have = (int)(cols - c < 4 ? cols - c : 4);
    const float f = e.column(c, have), scale[4] = {f, f, f, f};
    float x[FEW_D_W][4];
#pragma unroll
    for (int t = 0; t < FEW_D_W; ++t) {
        u32x2 four = {0, 0};
        if (t < n) four = *reinterpret_cast<const u32x2 *>(h + t * ldh + c); // rows of whole pieces of eight
        x[t][0] = bf16_lo(four[0]), x[t][1] = bf16_hi(four[0]), x[t][2] = bf16_lo(four[1]), x[t][3] = bf16_hi(four[1]);
    }
    for (int64_t v = v0; v < words && v < v0 + D_W_WORDS; v += 8) {
        float4 more[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (v + j < words) more[j] = get4(e.add, v + j, c, have);
        float sum[8][4] = {};
#pragma unroll
        for (int t = 0; t < FEW_D_W; ++t) {
            if (t >= n) break;
            const u32x4 z = *reinterpret_cast<const u32x4 *>(dz + t * ld + v); // dz's rows too
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float of = j & 1 ? bf16_hi(z[j >> 1]) : bf16_lo(z[j >> 1]);
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[j][k] = fmaf(of, x[t][k], sum[j][k]);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (v + j < words) put4(e.to, v + j, c, have, scale, make_float4(sum[j][0], sum[j][1], sum[j][2], sum[j][3]), more[j]);
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------------------
// The three products of a piece of the vocabulary.
plan16_t logits_plan(int64_t T, int64_t words, int64_t D) { return plan16(T, words, align_up(D, 8), false, 1); }
plan16_t d_h_plan(int64_t T, int64_t words, int64_t D) { return plan16(T, D, words, false); }
plan16_t d_w_plan(int64_t T, int64_t words, int64_t D) { return plan16(words, D, T, false); }

constexpr int64_t PIECE_BYTES = (int64_t)1 << 30; // of dz in the workspace, at most (one word's column however long)

bool copies_as_it_is(const adahop_tensor_t &x, int64_t cols) { return aligned(x.data, 16) && x.ld % 8 == 0 && cols % 8 == 0; }

struct forward_plan_t {
    int64_t tiles; // of whose words a token has numbers
    int few;       // k_ce_few's workgroups, or 0
    int64_t large; // words that large tiles are computed of, the first ones
    size_t part, at, h, w, total;
};

struct backward_plan_t {
    int64_t words, pieces, ld; // of a piece of the vocabulary
    size_t dz, sum_h, part, count, token, rows, h, w, total;
};

constexpr int64_t FEW_LDS = 64 * 1024; // of h: two workgroups on a compute unit, without an attribute

// Time of the logits of V words by tiles of either size, as plan16 sees it; a tile of 128 that has a compute unit to itself is of four waves here and takes 0.3 for half a slab.
double time_of_logits(int64_t T, int64_t V, int64_t D, bool large)
{
    const int64_t edge = large ? 256 : 128, room = large ? 256 : 512, tiles = ceil_div(T, edge) * ceil_div(V, edge), half_slabs = ceil_div(D, SLAB) * 2, rest = tiles % room;
    const double ends = large ? 12.0 : 6.0, each = (large ? 0.74 : 0.6) * (double)half_slabs;
    return (double)(tiles / room) * (ends + each) + (rest == 0 ? 0.0 : ends + (!large && rest <= 256 ? 0.3 * (double)half_slabs : each));
}

// Large tiles for all words, for none, or for as many as make whole rounds of them (50021 words for 1003 tokens of 2048: 213 us with large ones alone, four rounds of which the last has 16
// tiles).
int64_t words_of_large_tiles(int64_t T, int64_t V, int64_t D)
{
    const int64_t across = ceil_div(T, 256), rounds = across * ceil_div(V, 256) / 256, whole = rounds * 256 / across * 256;
    const double all = time_of_logits(T, V, D, true), none = time_of_logits(T, V, D, false);
    const double some = rounds > 0 && whole < V ? time_of_logits(T, whole, D, true) + time_of_logits(T, V - whole, D, false) + 3.0 : all;
    return some < all && some < none ? whole : all <= none ? V : 0;
}

// lay_h, lay_w: the operand is laid out anew
forward_plan_t forward_plan(int64_t T, int64_t V, int64_t D, bool lay_h, bool lay_w)
{
    forward_plan_t p;
    p.large = words_of_large_tiles(T, V, D);
    p.tiles = ceil_div(p.large, tile256_t::TM) + ceil_div(V - p.large, tile128_t::TM);
    p.few = 0;
    if (T <= FEW && (T <= 1 ? 1 : T <= 2 ? 2 : T <= 4 ? 4 : 8) * align_up(D, 512) * 2 <= FEW_LDS) {
        p.few = (int)(ceil_div(V, 16) < 512 ? ceil_div(V, 16) : 512); // two workgroups of four waves per compute unit
        p.tiles = p.few;
    }
    const size_t ld = align_up(D, 8) * 2;
    p.part = 0;
    p.at = align_up((size_t)T * p.tiles * sizeof(float2), 256);
    p.h = align_up(p.at + T * sizeof(float), 256);
    p.w = align_up(p.h + (lay_h ? T * ld : 0), 256);
    p.total = align_up(p.w + (lay_w ? V * ld : 0), 256);
    return p;
}

size_t most(size_t a, size_t b) { return a > b ? a : b; }

backward_plan_t backward_plan(int64_t T, int64_t V, int64_t D, bool lay_w)
{
    backward_plan_t p;
    const int64_t fit = PIECE_BYTES / 2 / T / 256 * 256, each = fit < 256 ? 256 : fit;
    p.pieces = ceil_div(V, each);
    p.words = p.pieces == 1 ? V : align_up(ceil_div(V, p.pieces), 256);
    p.pieces = ceil_div(V, p.words);
    p.ld = align_up(p.words, 8);
    const size_t ld = align_up(D, 8) * 2;
    const int64_t rest = V - (p.pieces - 1) * p.words;
    size_t part = 0;
    for (const int64_t words : {p.words, rest}) part = most(part, most(d_h_plan(T, words, D).part_bytes, d_w_plan(T, words, D).part_bytes));
    p.dz = 0;
    p.sum_h = align_up((size_t)T * p.ld * 2, 256);
    p.part = align_up(p.sum_h + (p.pieces > 1 ? (size_t)T * D * sizeof(float) : 0), 256);
    p.count = align_up(p.part + part, 256);
    p.token = p.count + 256;
    p.rows = align_up(p.token + T * sizeof(int32_t), 256);
    p.h = align_up(p.rows + T * sizeof(token_t), 256);
    p.w = align_up(p.h + T * ld, 256);
    p.total = align_up(p.w + (lay_w ? V * ld : 0), 256);
    return p;
}

device_once_t g_once;

template <class K> int launch_stats(product_t &q, const stats_t &e, hipStream_t st)
{
    q.nt = (uint32_t)ceil_div(q.A.outer, K::TM), q.dt = (uint32_t)ceil_div(q.B.outer, K::TN);
    k_ce_stats<K><<<q.nt * q.dt, K::THREADS, K::LDS, st>>>(q, e);
    return check_launch();
}

// h or w as the products take it: itself, or a copy at `to`.
int lay_out(const adahop_tensor_t &x, int64_t rows, int64_t cols, bool anew, void *to, side_t *out, hipStream_t st)
{
    if (!anew) {
        *out = {static_cast<const uint16_t *>(x.data), x.ld, rows};
        return ADAHOP_OK;
    }
    const int64_t ld = align_up(cols, 8), blocks = ceil_div(rows * (ld / 8), 256);
    *out = {static_cast<const uint16_t *>(to), ld, rows};
    k_lay_out<<<(unsigned)(blocks < 16384 ? blocks : 16384), 256, 0, st>>>(x, rows, cols, static_cast<uint16_t *>(to), ld);
    return check_launch();
}

} // namespace

int configure_linear_ce()
{
    int dev = 0;
    int rc = check_hip(hipGetDevice(&dev));
    if (rc != ADAHOP_OK || !g_once.need(dev)) return rc;
    rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void *>(&k_ce_stats<tile256_t>), hipFuncAttributeMaxDynamicSharedMemorySize, tile256_t::LDS));
    if (rc == ADAHOP_OK) rc = check_hip(hipFuncSetAttribute(reinterpret_cast<const void *>(&k_ce_stats<tile128_t>), hipFuncAttributeMaxDynamicSharedMemorySize, tile128_t::LDS));
    if (rc == ADAHOP_OK) rc = configure_all16<false, ALONG, ALONG, false, false, dlogits_t>();
    if (rc == ADAHOP_OK) rc = configure_all16<false, DOWN, DOWN, false, false, grad_t>();
    if (rc == ADAHOP_OK) rc = configure_all16<false, ALONG, DOWN, false, false, grad_t>();
    if (rc == ADAHOP_OK) g_once.mark(dev);
    return rc;
}

size_t linear_ce_workspace_bytes(const adahop_linear_ce_t &q, bool backward)
{
    const bool lay_h = !copies_as_it_is(q.h, q.dim), lay_w = !copies_as_it_is(q.w, q.dim);
    return backward ? backward_plan(q.tokens, q.vocab, q.dim, lay_w).total : forward_plan(q.tokens, q.vocab, q.dim, lay_h, lay_w).total;
}

void linear_ce_plan(int64_t T, int64_t V, int64_t D, int product, int *tile, int *alone, int *slices)
{
    const int64_t words = backward_plan(T, V, D, false).words;
    if (product == 2 && T <= FEW_D_W) {
        *tile = 0, *alone = 0, *slices = 1;
        return;
    }
    const plan16_t p = product == 0 ? logits_plan(T, words, D) : product == 1 ? d_h_plan(T, words, D) : d_w_plan(T, words, D);
    *tile = p.edge, *alone = alone16(p), *slices = (int)p.slices;
}

int launch_linear_ce(const adahop_linear_ce_t &c, void *workspace, hipStream_t st)
{
    int rc = configure_linear_ce();
    if (rc != ADAHOP_OK) return rc;
    const bool lay_h = !copies_as_it_is(c.h, c.dim), lay_w = !copies_as_it_is(c.w, c.dim);
    const forward_plan_t p = forward_plan(c.tokens, c.vocab, c.dim, lay_h, lay_w);
    char *const ws = static_cast<char *>(workspace);
    product_t q = {};
    if ((rc = lay_out(c.w, c.vocab, c.dim, lay_w, ws + p.w, &q.A, st)) != ADAHOP_OK) return rc;
    if ((rc = lay_out(c.h, c.tokens, c.dim, lay_h, ws + p.h, &q.B, st)) != ADAHOP_OK) return rc;
    q.K = align_up(c.dim, 8);
    stats_t e = {{c.targets, c.tokens, c.vocab, c.logit_scale, c.z_loss}, 0, 0, p.tiles, reinterpret_cast<float2 *>(ws + p.part), reinterpret_cast<float *>(ws + p.at)};
    if (p.few) {
        const int room = c.tokens <= 1 ? 1 : c.tokens <= 2 ? 2 : c.tokens <= 4 ? 4 : 8;
        const size_t lds = (size_t)room * align_up(c.dim, 512) * 2;
        switch (room) {
        case 1: k_ce_few<1><<<p.few, 256, lds, st>>>(q.A, q.B, q.K, e); break;
        case 2: k_ce_few<2><<<p.few, 256, lds, st>>>(q.A, q.B, q.K, e); break;
        case 4: k_ce_few<4><<<p.few, 256, lds, st>>>(q.A, q.B, q.K, e); break;
        default: k_ce_few<8><<<p.few, 256, lds, st>>>(q.A, q.B, q.K, e);
        }
        rc = check_launch();
    } else {
        q.A.outer = p.large;
        if (p.large > 0 && (rc = launch_stats<tile256_t>(q, e, st)) != ADAHOP_OK) return rc;
        q.A.data += p.large * q.A.ld, q.A.outer = c.vocab - p.large;
        e.v0 = p.large, e.tile = ceil_div(p.large, tile256_t::TM);
        if (q.A.outer > 0) rc = launch_stats<tile128_t>(q, e, st);
    }
    if (rc != ADAHOP_OK) return rc;
    k_ce_join<<<(unsigned)ceil_div(c.tokens, 4), 256, 0, st>>>(e.p, e.part, e.at, (int)p.tiles, c.loss, c.lse);
    return check_launch();
}

int launch_linear_ce_backward(const adahop_linear_ce_t &c, void *workspace, hipStream_t st)
{
    int rc = configure_linear_ce();
    if (rc != ADAHOP_OK) return rc;
    const bool lay_w = !copies_as_it_is(c.w, c.dim);
    const int64_t T = c.tokens, V = c.vocab, D = c.dim, ldh = align_up(D, 8);
    const backward_plan_t p = backward_plan(T, V, D, lay_w);
    char *const ws = static_cast<char *>(workspace);
    int32_t *const count = reinterpret_cast<int32_t *>(ws + p.count), *const token = reinterpret_cast<int32_t *>(ws + p.token);
    uint16_t *const dz = reinterpret_cast<uint16_t *>(ws + p.dz), *const h = reinterpret_cast<uint16_t *>(ws + p.h);
    token_t *const rows = reinterpret_cast<token_t *>(ws + p.rows);
    side_t w;
    if ((rc = lay_out(c.w, V, D, lay_w, ws + p.w, &w, st)) != ADAHOP_OK) return rc;
    k_ce_tokens<<<1, 1024, 0, st>>>(c.targets, T, token, count);
    if ((rc = check_launch()) != ADAHOP_OK) return rc;
    const bool one = !c.d_loss || c.d_loss_stride == 0; // d_loss for all tokens
    const float factor = one ? c.logit_scale : 1.0f;
    const float *const by = one ? c.d_loss : nullptr;
    k_gather<<<(unsigned)T, 256, 0, st>>>(c.h, D, {c.targets, T, V, c.logit_scale, c.z_loss}, c.lse, one ? nullptr : c.d_loss, c.d_loss_stride, one ? 1.0f : c.logit_scale, token, count, h,
                                          ldh, rows);
    if ((rc = check_launch()) != ADAHOP_OK) return rc;
    if (c.d_h.data) {
        k_ce_zeros<<<(unsigned)T, 256, 0, st>>>(c.targets, D, c.d_h);
        if ((rc = check_launch()) != ADAHOP_OK) return rc;
    }
    const adahop_tensor_t none = {}, sum_h = {ws + p.sum_h, D, 1};
    for (int64_t i = 0; i < p.pieces; ++i) {
        const int64_t v0 = i * p.words, words = V - v0 < p.words ? V - v0 : p.words, ld = align_up(words, 8);
        const side_t piece = {w.data + v0 * w.ld, w.ld, words};
        product_t q = {};
        q.A = {h, ldh, T}, q.B = piece, q.K = ldh;
        q.rows_of = count;
        const dlogits_t e = {rows, c.logit_scale, c.z_loss, v0, words, ld, dz};
        if ((rc = launch_product16<false, ALONG, ALONG, false, false>(logits_plan(T, words, D), q, e, nullptr, st)) != ADAHOP_OK) return rc;
        if (c.d_h.data) { // first: what the caches still hold of w is of use (15 tokens of 4096, 65536 words: 476 us, 491 behind d_w)
            const bool end = i + 1 == p.pieces;
            q.A = {dz, ld, T}, q.B = {piece.data, piece.ld, D}, q.K = words;
            q.rows_of = count, q.K_of = nullptr;
            const grad_t g = {end ? c.d_h : sum_h, i ? sum_h : none, end ? token : nullptr, factor, by, count};
            if ((rc = launch_product16<false, ALONG, DOWN, false, false>(d_h_plan(T, words, D), q, g, ws + p.part, st)) != ADAHOP_OK) return rc;
        }
        if (c.d_w.data) {
            const int64_t size = c.d_w.f32 ? 4 : 2, size_add = c.add.f32 ? 4 : 2;
            q.A = {dz, ld, words}, q.B = {h, ldh, D}, q.K = T;
            q.rows_of = nullptr, q.K_of = count;
            const grad_t g = {{static_cast<char *>(c.d_w.data) + v0 * c.d_w.ld * size, c.d_w.ld, c.d_w.f32},
                              c.add.data ? adahop_tensor_t{static_cast<char *>(c.add.data) + v0 * c.add.ld * size_add, c.add.ld, c.add.f32} : none, nullptr, factor, by, count};
            if (T <= FEW_D_W) {
                k_ce_d_w_few<<<dim3((unsigned)ceil_div(words, D_W_WORDS), (unsigned)ceil_div(D, 1024)), 256, 0, st>>>(h, ldh, dz, ld, count, words, D, g);
                rc = check_launch();
            } else
                rc = launch_product16<false, DOWN, DOWN, false, false>(d_w_plan(T, words, D), q, g, ws + p.part, st);
            if (rc != ADAHOP_OK) return rc;
        }
    }
    return ADAHOP_OK;
}

// d_w = add, or 0, where there are no tokens.
__global__ __launch_bounds__(256) void k_ce_no_tokens(adahop_tensor_t to, adahop_tensor_t add, int64_t rows, int64_t cols)
{
    const int64_t c = ((int64_t)blockIdx.y * 64 + (threadIdx.x & 63)) * 4, r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (c >= cols || r >= rows) return;
    const int have = (int)(cols - c < 4 ? cols - c : 4);
    const float one[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    put4(to, r, c, have, one, make_float4(0.0f, 0.0f, 0.0f, 0.0f), get4(add, r, c, have));
}

int launch_linear_ce_no_tokens(const adahop_linear_ce_t &c, hipStream_t st)
{
    k_ce_no_tokens<<<dim3((unsigned)ceil_div(c.vocab, 4), (unsigned)ceil_div(c.dim, 256)), 256, 0, st>>>(c.d_w, c.add, c.vocab, c.dim);
    return check_launch();
}

} // namespace adahop

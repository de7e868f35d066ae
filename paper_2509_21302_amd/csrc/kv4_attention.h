// What the kernels of attention over the 4-bit key/value cache share: a wave's way through the pages, and its rows.
//
//     o = softmax_j(scale <q, k_j>) v_j,   k_j = step (code_j H) s,  v_j likewise:   <q, k_j> = step <(s q) H, code_j>,   o = s ((sum_j p_j step_j code_j) H)
//
// so queries are turned once, products are taken with the codes themselves, a token's step is a factor of its score or its weight, and the sum is turned back at the end.
//
// The codes go to the matrix cores as fp16 numbers without a conversion: u = code + 8 in the low four bits of a half word is the subnormal u 2^-24, one nibble
// up it is 16 u 2^-24, both exact (the instruction does not flush them), so a word of 8 codes is four operands after one shift and four ands.  The 16 of the odd channels is taken
// out of the queries in the one product and out of the sum in the other, and the 8 that every code is too large by comes off in the accumulator that the first product starts from
// and, in the second, every few hundred steps with the sum of the weights that one more instruction on eights makes.  Queries are fp16 with a power of two common to a wave, weights fp16 scaled so
// that they reach down to 2^-31 of the largest: 11 bits, against 8 of a bf16 that the result is rounded to.
//
// A wave takes 32 tokens a step: scores of 32 tokens x 16 rows (keys x queries), exp2, weights, sums (values x weights) -- the accumulators of the first product have, lane by lane, the
// tokens that the second product's operand needs, so nothing moves between lanes.  Rows are the query tokens of a sequence times the query heads that share a key head.
#pragma once
#include "kv4.h"

namespace qvggt {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

union Operand {                 // eight fp16 numbers of a lane
    uint32_t w[4];
    half8 h;
};

// Two numbers, each to the nearest fp16, in one instruction.  (Cut off, they would be 2^-12 too small on average against the sum of weights that results are divided by.)
__device__ inline uint32_t nearest_fp16(float a, float b)
{
    typedef float Two __attribute__((ext_vector_type(2)));
    typedef _Float16 TwoHalves __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((Two{a, b}), TwoHalves));
}

__device__ inline float4v mfma(const Operand &a, const Operand &b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, b.h, c, 0, 0, 0); }

constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -1e30f;                 // running maximum of a row that has seen nothing
constexpr float kSlack = 8.0f;                  // weights may pass 1 by this many powers of two before sums are scaled down
constexpr int kTop = 7;                         // log2 of a weight at the running maximum with the largest step: 2^15 with the slack, under fp16's 65504
constexpr int kSmallest = -90;                  // log2 of the least largest step that weights are scaled up for (fp32 sums of 2^20 of them stay in range)

// what a block knows about its sequence
struct Sequence {
    int start, n, len;      // queries and keys, cut off at what the caller states as their most
    int before;             // keys in front of the first query's own, of the whole sequence (or the most keys, where there are more): what is cut off must not shift what a query sees
};
__device__ inline Sequence sequence_of(const Kv4Attention &a, int b)
{
    Sequence s;
    s.start = min(max(a.starts[b], 0), a.T);
    const int n = max(min(a.starts[b + 1], a.T) - s.start, 0), len = max(a.lens[b], 0);
    s.n = min(n, a.max_q);
    s.len = min(len, a.max_kv);
    s.before = min(len - n, a.max_kv);
    return s;
}
// keys that a query token sees
__device__ inline int visible(const Kv4Attention &a, const Sequence &s, int token) { return a.causal ? min(max(s.before + token + 1, 0), s.len) : s.len; }

// floats of a row's partial sums: D sums, the maximum, the sum of weights
template <int D>
constexpr int kPartial = D + 2;

// A row's sums (16 lanes) over its weights, turned back and written.  No weights: zeros; weights that are no number stay none.
template <int D>
__device__ inline void finish_row(const Kv4Attention &a, int group, const Sequence &s, int head, int row, float (&x)[D / 16], float total, int lane)
{
    constexpr int C = D / 16;
    const int first = (lane & 15) * C;
    const float factor = total > 0.0f || total != total ? kv4_norm<D>() / total : 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] *= factor;
    row_butterflies<C>(x, lane);
    sign_channels<C>(a.signs, first, x);
    uint16_t *to = a.out + ((size_t)(s.start + row / group) * a.q_heads + head * group + row % group) * D + first;
#pragma unroll
    for (int i = 0; i < C / 4; ++i) reinterpret_cast<uint2 *>(to)[i] = make_uint2(pack_bf16x2(x[4 * i], x[4 * i + 1]), pack_bf16x2(x[4 * i + 2], x[4 * i + 3]));
}
template <int D>
__device__ inline void leave_row(float *to, const float (&x)[D / 16], float top, float total, int lane)
{
    constexpr int C = D / 16;
#pragma unroll
    for (int i = 0; i < C / 2; ++i) reinterpret_cast<float2 *>(to + (lane & 15) * C)[i] = make_float2(x[2 * i], x[2 * i + 1]);
    if ((lane & 15) == 0) *reinterpret_cast<float2 *>(to + D) = make_float2(top, total);
}

// The way of a wave through a sequence's pages.  It holds AHEAD steps of 32 tokens: a step's registers are filled with the one AHEAD steps on as soon as they are taken apart, its
// pages are looked up (scalar loads) a step before that.  Blocks of 16 tokens behind the last one are taken as the last one.
template <int D, int AHEAD, bool ONCE>
struct Keys {
    using L = Kv4Layout<D>;
    static constexpr int W = L::kWords;
    typedef const __attribute__((address_space(4))) int32_t *Table;
    Table table;
    const uint8_t *head_base;
    size_t page_bytes;
    int page_shift, page_mask, num_pages, last_block;
    uint32_t key_of_lane, value_of_lane, step_of_lane;
    int page[2], at[2];             // of the step after the one that is fetched; of the one that is
    const uint8_t *part[2];
    uint32_t k[AHEAD][2][W], v[AHEAD][2][W], s[AHEAD][2][4];

    __device__ void find(int t0)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) page[h] = table[min(t0 / 16 + h, last_block) * 16 >> page_shift];
    }
    __device__ void locate(int t0)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            at[h] = min(t0 / 16 + h, last_block) * 16 & page_mask;
            part[h] = head_base + (size_t)min(max(page[h], 0), num_pages - 1) * page_bytes;
        }
    }
    // ONCE: the caches need not keep these bytes, which nobody else reads (or one block more, where a head has two tiles of rows in shared blocks: it reads memory again)
    template <int N>
    __device__ static void words(const uint8_t *base, uint32_t offset, uint32_t (&w)[N])
    {
        // 64 channels: the offset beside an address in scalar registers.  Left alone, the compiler keeps it as 64 bits across the loop and adds them, six registers more, and four tiles spill
        // (a frame over 50: 620 us, 643 without).  128 channels have the room, and the additions cost nothing there
        if (D == 64) asm("" : "+v"(offset) : "s"((uint32_t)(uintptr_t)base));
        const uint8_t *const from = base + offset;
        typedef uint32_t Vector __attribute__((ext_vector_type(N)));
        const Vector x = ONCE ? __builtin_nontemporal_load(reinterpret_cast<const Vector *>(from)) : *reinterpret_cast<const Vector *>(from);
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = x[i];
    }
    __device__ void fetch_keys(int d, int h) { words(part[h] + L::keys(at[h]), key_of_lane, k[d][h]); }
    __device__ void fetch_values(int d, int h) { words(part[h] + L::values(at[h], page_shift), value_of_lane, v[d][h]); }
    __device__ void fetch_steps(int d, int h) { words(part[h] + L::steps(at[h], page_shift), step_of_lane, s[d][h]); }
    // the first step at t0 (a step at which there is something), the others `stride` tokens apart
    __device__ void begin(const Kv4Attention &a, int b, int head, int last, int t0, int stride, int lane)
    {
        table = reinterpret_cast<Table>(reinterpret_cast<uintptr_t>(a.table + (size_t)b * a.table_width));
        page_shift = a.pages.page_shift;
        page_mask = (1 << page_shift) - 1;
        num_pages = a.pages.num_pages;
        page_bytes = a.pages.heads * ((size_t)(D + 4) << page_shift);
        head_base = a.pages.base + head * ((size_t)(D + 4) << page_shift);
        last_block = (last - 1) / 16;
        key_of_lane = (lane & 15) * L::kRow + (lane >> 4) * 4 * W;
        value_of_lane = lane * 4 * W;
        step_of_lane = (lane >> 4) * 16;
        int first[AHEAD][2];
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            find(t0 + d * stride);
            first[d][0] = page[0];
            first[d][1] = page[1];
        }
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            page[0] = first[d][0];
            page[1] = first[d][1];
            locate(t0 + d * stride);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                fetch_keys(d, h);
                fetch_steps(d, h);
                fetch_values(d, h);
            }
        }
        find(t0 + AHEAD * stride);
    }
};

// 16 NT rows of a wave: queries as operands, running maxima, sums.
template <int D, int NT, int AHEAD, bool ONCE>
struct Rows {
    static constexpr int C = D / 16, W = D / 32, S = D / 32;
    static constexpr int kPad = D + 4;  // floats of a row in LDS
    Operand q[NT][S];
    float base[NT];                     // what the first product starts from: -8 times the sum of the queries
    int end[NT];                        // keys that the lane's row sees
    int exponent[NT];                   // log2 of a tile's unit
    float unit;                         // of the product of a query number and a subnormal: 1 .. 2^27
    // Weights are 2^(score - m): m is the running maximum less the row's lift, by which weights times steps fill fp16's range (kTop below the top at a step that is the power of two above
    // all steps of values that the row has seen; a row's own, so that nothing depends on values that only its neighbours see).  l: their sum; acc, ones: their sums times step times code + 8,
    // and times step times 8.  Whatever the lift, sums over l are the result.
    float4v acc[NT][2 * W], ones[NT];
    float m[NT], l[NT];
    float *lifts;                       // of the wave's rows, in LDS: [tile][row]
    float reach, low;                   // of all rows: the least power of two, the least lift
    uint32_t seen;                      // bit j: the lane's row of tile j has a maximum (or will never have one)
    float unseen;                       // infinite until all have

    // A row of queries on its way to LDS: what 16 lanes load of it (rows behind the last one: the last one), and the row turned.
    struct Query {
        HeadRow<C> x;
        __device__ void load(const Kv4Attention &a, const Sequence &seq, int head, int group, int row, int rows, int lane)
        {
            const int r = min(row, rows - 1), token = r / group, first = (lane & 15) * C;
            const void *from = static_cast<const char *>(a.q) + ((seq.start + token) * a.q_stride + (long long)(head * group + r - token * group) * D) * (a.q_f32 ? 4 : 2);
            x.load(from, a.q_f32, first, a.signs);
            x.load_turn(from, a.q_f32, first, a.rope, seq.start + token);
        }
        __device__ void load_angles(const Kv4Attention &a, int lane) { x.load_angles((lane & 15) * C, a.rope); }
        __device__ void store(const Kv4Attention &a, bool there, float *turned, int lane) const
        {
            const int first = (lane & 15) * C;
            float y[C];
            x.turned(a.q_f32, first, a.rope, a.signs, y);
            row_butterflies<C>(y, lane);
            const float f = there ? kv4_norm<D>() * a.scale * kLog2e : 0.0f;
#pragma unroll
            for (int i = 0; i < C; ++i) turned[first + i] = there ? y[i] * f : 0.0f;
        }
    };
    // tile j's operands from 16 turned rows in LDS.  Lane (n, g) has channels g D / 4 .. of row n, as the keys' lanes have
    __device__ void take_queries(int j, const float *turned, int lane)
    {
        float x[D / 4], top = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 4; ++i) {
            x[i] = turned[(lane & 15) * kPad + (lane >> 4) * (D / 4) + i];
            top = fmaxf(top, fabsf(x[i]));
        }
        top = max_over_64_lanes(top);
        // 2^(13 - e) with 2^e <= top < 2^(e + 1): the largest query number of the tile in 2^13 .. 2^14, the others to an absolute error that is 2^-25 of a score unit at least.
        // Numbers over 2^19 (scores in the hundred thousands at least: one key takes all the weight) become the largest fp16 and leave the other rows alone; infinities and no numbers stay
        const int e = min(max((int)(__float_as_uint(top) >> 23), 127 - 11), 127 + 16);
        exponent[j] = e - 127 - 13;
        const float up = __uint_as_float((uint32_t)(127 + 13 - (e - 127)) << 23);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[i] = x[8 * s + i] * up;
                y[i] = fabsf(y[i]) < INFINITY ? __builtin_amdgcn_fmed3f(y[i], -65504.0f, 65504.0f) : y[i];
                if (i & 1) y[i] *= 0.0625f;
            }
            constexpr int order[8] = {0, 4, 1, 5, 2, 6, 3, 7};
#pragma unroll
            for (int i = 0; i < 8; ++i) q[j][s].h[i] = (_Float16)y[order[i]];
        }
    }
    __device__ int highest_exponent() const
    {
        int highest = exponent[0];
#pragma unroll
        for (int j = 1; j < NT; ++j) highest = max(highest, exponent[j]);
        return highest;
    }
    // all tiles on one power of two, and nothing seen yet
    __device__ void start(int highest, float *room)
    {
        lifts = room;
        unit = __uint_as_float((uint32_t)(highest + 24 + 127) << 23);
        const float4v zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const _Float16 down = (_Float16)__builtin_amdgcn_exp2f((float)(exponent[j] - highest));
            float sum = 0.0f;
#pragma unroll
            for (int s = 0; s < S; ++s)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q[j][s].h[i] = q[j][s].h[i] * down;
                    sum += (float)q[j][s].h[i] * ((i >> 1) & 1 ? 16.0f : 1.0f);
                }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            base[j] = -sum * 0x1p-21f;
#pragma unroll
            for (int c = 0; c < 2 * W; ++c) acc[j][c] = zero;
            ones[j] = zero;
            m[j] = l[j] = 0.0f;
        }
        reach = low = 0.0f;
#pragma unroll
        for (int j = 0; j < NT; ++j) lifts[16 * j + row_of_lane()] = kTop - kSmallest;
        seen = 0;
#pragma unroll
        for (int j = 0; j < NT; ++j) seen |= (uint32_t)(end[j] == 0) << j;
        unseen = INFINITY;
    }
    // The lane's row of a tile, without a register of its own beside the loops
    __device__ static int row_of_lane()
    {
        unsigned none = 0;
        asm volatile("" : "+s"(none));
        return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none)) & 15;
    }
    // t: the scores of a step above m, -inf where a row does not see a key.  Where one is above the maximum by more than the slack, a value's step above all that some row has seen, or a row
    // without a maximum: maxima and lifts anew, and t and the sums with them.  (Scores are got back from t: nothing else of the step is kept for this.)
    __device__ void raise(float (&t)[NT][2][4], const float (&vs)[2][4], float over, float tops)
    {
        if (!__builtin_amdgcn_ballot_w64(over > kSlack + low || tops > reach)) return;
        float lowest = kTop - kSmallest, highest = kTop - 127;
        float *const mine = lifts + row_of_lane();
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            float top = -INFINITY, loud = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    top = fmaxf(top, t[j][h][i]);
                    loud = fmaxf(loud, t[j][h][i] > -INFINITY ? vs[h][i] : 0.0f);
                }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            loud = fmaxf(loud, __shfl_xor(loud, 16));
            loud = fmaxf(loud, __shfl_xor(loud, 32));
            const float before = mine[16 * j], lift = fminf(before, (float)(kTop - max((int)(__float_as_uint(loud) >> 23) - 126, kSmallest)));          // (2^(kTop - lift) > loud)
            const bool first = !(seen >> j & 1), any = top > -INFINITY;
            const float up = first ? (any ? top - lift : 0.0f) : fmaxf(top, before) - lift;                 // (t has the lift in it)
            const float down = first ? 1.0f : __builtin_amdgcn_exp2f(-up);                    // (a first maximum: there are no sums yet)
            mine[16 * j] = lift;                // (each lane reads back what it wrote)
            seen |= (uint32_t)any << j;
            m[j] += up;
            l[j] *= down;
            if (end[j] != 0) highest = fmaxf(highest, lift);
            lowest = fminf(lowest, lift);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) t[j][h][i] -= up;
            ones[j] *= down;
#pragma unroll
            for (int c = 0; c < 2 * W; ++c) acc[j][c] *= down;
        }
        low = -__int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(max_over_64_lanes(-lowest))));      // (scalars)
        reach = __uint_as_float((uint32_t)(kTop + 127 - (int)__int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(max_over_64_lanes(highest))))) << 23);
        unseen = seen == (1u << NT) - 1 ? kNone : INFINITY;
    }
    // A tile's weights of 32 keys from their scores above m: their sum, and with the values' steps the operand of the second product.  Tokens 0, 2 and 1, 3 of a group of four lie
    // together, as the bytes of a value's word come apart.  EDGE: a key that the row does not see counts nothing, whatever its step is (0 times a step that is no number is none).
    template <bool EDGE>
    __device__ void weigh(int j, const float (&t)[2][4], const float (&vs)[2][4], Operand &p)
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float e[4], w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e[i] = __builtin_amdgcn_exp2f(t[h][i]);
                w[i] = EDGE && t[h][i] == -INFINITY ? 0.0f : e[i] * vs[h][i];
            }
            l[j] += (e[0] + e[1]) + (e[2] + e[3]);
            p.w[2 * h] = nearest_fp16(w[0], w[2]);
            p.w[2 * h + 1] = nearest_fp16(w[1], w[3]);
        }
    }
    // The offset of 8 out of the sums so far.  It grows with every key, what is left of the sums without it (values of both signs) much less, and every addition is rounded at the size of the
    // whole: over 2^20 keys of the same weight in one wave 1.7 % of the result, and below 10^-4 where the offset starts anew every kFold steps
    static constexpr int kFold = 256;
    __device__ void fold()
    {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                acc[j][2 * w] -= ones[j];
                acc[j][2 * w + 1] -= 16.0f * ones[j];
            }
            ones[j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
    // The 32 keys from t0, which `x` holds in place d, and the fetch of those AHEAD steps on.  EDGE: some row does not see all of them; last: keys that some row sees.
    template <bool EDGE>
    __device__ void take(Keys<D, AHEAD, ONCE> &x, int d, int t0, int stride, int last, int g)
    {
        float ks[2][4], vs[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // (a product and not a sum of exponents, which is an instruction less and 1 to 2 % of a prompt: a step that is no number stays none)
                ks[h][i] = __uint_as_float(x.s[d][h][i] << 16) * unit;
                vs[h][i] = __uint_as_float(x.s[d][h][i] & 0xffff0000u);
                if (EDGE && t0 + 16 * h + 4 * g + i >= last) vs[h][i] = 0.0f;             // behind the end lies whatever was there: no number, perhaps
            }
        x.locate(t0 + AHEAD * stride);
        x.find(t0 + (AHEAD + 1) * stride);
        // scores, in powers of two above the running maximum
        float4v sc[NT][2];
        float t[NT][2][4], over = unseen, tops = 0.0f;
        auto product = [&](int h, int s) {
            Operand k;
            const uint32_t w = x.k[d][h][s], u = w >> 8;
            k.w[0] = w & kLow; k.w[1] = w & kHigh; k.w[2] = u & kLow; k.w[3] = u & kHigh;
#pragma unroll
            for (int j = 0; j < NT; ++j) sc[j][h] = mfma(k, q[j][s], s == 0 ? float4v{base[j], base[j], base[j], base[j]} : sc[j][h]);
        };
        // One tile: the two blocks in turn, a product need not wait for the one before (64 sequences to 8192 keys 76 -> 69 us); several tiles are turns enough, and block after
        // block lets go of registers earlier (prompt of 12289 tokens 1.29 ms, 1.32 the other way)
        if constexpr (NT == 1) {
#pragma unroll
            for (int s = 0; s < S; ++s) {
                product(0, s);
                product(1, s);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (NT > 1) {
#pragma unroll
                for (int s = 0; s < S; ++s) product(h, s);
            }
            x.fetch_keys(d, h);
            x.fetch_steps(d, h);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                tops = fmaxf(tops, vs[h][i]);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    t[j][h][i] = fmaf(sc[j][h][i], ks[h][i], -m[j]);
                    if (EDGE && t0 + 16 * h + 4 * g + i >= end[j]) t[j][h][i] = -INFINITY;
                    over = fmaxf(over, t[j][h][i]);
                }
            }
        raise(t, vs, over, tops);
        Operand p[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) weigh<EDGE>(j, t[j], vs, p[j]);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            Operand low, high;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t v = x.v[d][h][w], u = v >> 8;
                low.w[2 * h] = v & kLow; low.w[2 * h + 1] = u & kLow;
                high.w[2 * h] = v & kHigh; high.w[2 * h + 1] = u & kHigh;
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                acc[j][2 * w] = mfma(low, p[j], acc[j][2 * w]);
                acc[j][2 * w + 1] = mfma(high, p[j], acc[j][2 * w + 1]);
            }
        }
        x.fetch_values(d, 0);
        x.fetch_values(d, 1);
        Operand eights;
#pragma unroll
        for (int i = 0; i < 4; ++i) eights.w[i] = 0x00080008u;
#pragma unroll
        for (int j = 0; j < NT; ++j) ones[j] = mfma(eights, p[j], ones[j]);
    }
    // The steps t0, t0 + stride, ... below stop; the first of them are below `full`, which every row sees.  (One loop with both kinds of step in it takes 70 registers more.)
    __device__ void run(Keys<D, AHEAD, ONCE> &x, int t0, int stride, int full, int last, int stop, int g)
    {
        for (const int whole = min(full, stop) - 32 - (AHEAD - 1) * stride; t0 <= whole;) {
            const int pause = min(whole, t0 | (kFold * stride - 1));
            for (; t0 <= pause; t0 += AHEAD * stride) {
#pragma unroll
                for (int d = 0; d < AHEAD; ++d) take<false>(x, d, t0 + d * stride, stride, last, g);
            }
            fold();                         // (a loop of its own around the steps: 2 % less than a branch within them)
        }
        for (; t0 < stop; t0 += AHEAD * stride) {
#pragma unroll
            for (int d = 0; d < AHEAD; ++d)
                if (d == 0 || t0 + d * stride < stop) take<true>(x, d, t0 + d * stride, stride, last, g);
        }
    }

    // tile j's sums to LDS, row by row (lane (n, g) has channels 2 W (4 g + i) + c of row n), with maxima and sums of weights
    __device__ void leave(int j, float *rows16, float *tops, float *totals, int lane)
    {
        const int n = lane & 15, g = lane >> 4;
        float total = l[j];
        total += __shfl_xor(total, 16);
        total += __shfl_xor(total, 32);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float *to = rows16 + n * kPad + 2 * W * (4 * g + i) + 2 * w;
                to[0] = (acc[j][2 * w][i] - ones[j][i]) * 0x1p24f;
                to[1] = (acc[j][2 * w + 1][i] * 0.0625f - ones[j][i]) * 0x1p24f;
            }
        if (g == 0) {
            tops[n] = seen >> j & 1 ? m[j] : kNone;
            totals[n] = total;
        }
    }
};

}  // namespace
}  // namespace qvggt

// Attention of packed sequences over bf16 keys and values:   out[i, h] = sum_j softmax_j(scale <q[i, h], k[j, h']>) v[j, h'].
//
// Rows are the query tokens of a sequence times the query heads that share a key head; a wave has tiles of M = 16 or 32 of them.  Scores are keys x queries and results channels x queries, both
// v_mfma_f32_16x16x32_bf16 or v_mfma_f32_32x32x16_bf16.  With G = 64 / M groups of lanes, group g of a lane, its accumulators of consecutive tiles of keys are the keys
//     number f  =  key 4 G (f / 4) + 4 g + f % 4
// of one row, and eight of them are what its part of the second product's right operand is made of, if the 8 G keys of a step come in that order in both operands.  So nothing moves between lanes but
// a maximum and a sum for every row, and a row's factor is a lane's.  The values' operand has that order from LDS reads that transpose: four keys of sixteen channels a group of sixteen lanes.
//
// Keys and values go straight from memory into LDS, 16 bytes a lane, rows as they are.  A row's 16-byte pieces change places by its number (the source address does that), so that reads
// of rows of keys, and of a few rows of values, touch every bank as often as any other.
//
// The running maximum of a row is raised when scores exceed it by much: weights are at most 2^8 or 2^12 then, which costs bf16 and fp32 nothing, and sums are multiplied by a factor in few steps.
// In the steps that all rows of a block see it is not even looked for: the sum of a step's weights says whether one of them is too large, and only then are they made again (what that saves is 12 %
// of the vector instructions: 13740 rows on as many keys, 16 heads x 64, 809 us for 856; 8192 on 8192, 16 x 128, 485 for 501).  Weights are rounded to bf16 (to nearest), for the product and for the sum
// that it is divided by alike.  A row starts from a maximum of the lowest number, so that rows that see nothing end with a sum of 0.
//
// A weight's exponent is one multiplication and addition, score * scale2 - maximum * scale2, as long as the second product is small: at 2^12 its rounding is 2^-13 of an exponent, at 2^31 whole weights, and past
// fp32 all of them.  Rows of larger ones have differences of scores instead, times the scale, which are right at any scale.  That is an instruction
// more a score, and in the steps that all rows see weights made twice, only where there are such rows (scores of +-20000: 13740 rows on as many keys, 16 heads x 64, 1167 us for 903 without; 11003 tokens, 32 heads on
// 8 x 128, 1119 for 997).
#include <type_traits>

#include "attention.h"
#include "attention_plan.h"
#include "lds_transfer.h"

namespace qvggt {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
union Operand {
    uint4 u;
    uint32_t w[4];
    short4v s[2];
    bf16x8 b;
};

constexpr float kNone = -3.4028235e38f, kLog2e = 1.4426950408889634f;       // kNone: the maximum that a row starts from
constexpr float kSlack = 8.0f, kMostWeights = 4096.0f;       // log2 of a weight; a lane's weights of a step, and the maximum * scale2 from which they are of differences

struct Cut {
    Attention a;
    int group, chunk, splits, tiles;        // query heads of a key head; keys of a part; parts and tiles of rows that there may be
    float scale2;                           // |scale| log2(e), 1 for a scale of 0; its sign, and a scale of 0, are in the queries
    uint32_t flip;                          // ... the sign as a mask of pairs of them
    int zero;                               // ... whether the scale is 0: queries of 0, or NaN where they are no numbers
    float *partials;                        // [seqs][key heads][rows][splits][D + 2]: a row's sums, maximum and weights' sum
};

// ---- a sequence
struct Sequence {
    int q0, n, k0;              // first row of the queries, how many are answered, first row of the keys
    int total, len, limit;      // queries and keys there are, keys that are looked at
};
__device__ inline Sequence sequence_of(const Attention &a, int b)
{
    Sequence s;
    s.q0 = min(max(a.q_starts[b], 0), a.T);
    s.total = min(max(a.q_starts[b + 1], s.q0), a.T) - s.q0;
    s.n = min(s.total, a.max_q);
    s.k0 = min(max(a.kv_starts[b], 0), a.S);
    s.len = min(max(a.kv_lens != nullptr ? a.kv_lens[b] : max(a.kv_starts[b + 1], 0) - s.k0, 0), a.S - s.k0);
    s.limit = min(s.len, a.max_kv);
    return s;
}
// Keys that query i sees.
__device__ inline int visible(const Attention &a, const Sequence &s, int i) { return a.causal ? min(max(s.len - s.total + i + 1, 0), s.limit) : s.limit; }
// What a row's sums are multiplied by.  A row without keys is zeros; the weights of one that sees keys add up to 0 where all its scores are -infinity, which have no softmax.
__device__ inline float share_of(float total, int seen) { return total != 0.0f ? 1.0f / total : seen > 0 ? __builtin_nanf("") : 0.0f; }

// ---- how rows lie in LDS
template <int D, int M>
struct Rows {
    static constexpr int kBytes = 2 * D, kPieces = D / 8, kPerTransfer = 64 / kPieces;      // rows that one transfer of a wave brings
    // Place of piece c of a row.  Of keys, sixteen lanes read as many rows at one piece; of values, thirty-two lanes read eight rows at two pieces (M = 16) or four rows at four
    __device__ static int key_piece(int row, int c) { return D == 128 ? c ^ (row & 15) : c ^ (row >> 1 & 7); }
    __device__ static int value_piece(int row, int c)
    {
        if (M == 16) return D == 128 ? c ^ (row & 7) << 1 : c ^ (row >> 1 & 3) << 1;
        return D == 128 ? c ^ (row & 3) << 2 : c ^ (row >> 1 & 1) << 2;
    }
};

// A pair of bf16 times 0.
__device__ inline uint32_t none_of(uint32_t w) { return ((w & 0x7f80u) == 0x7f80u ? 0x7fc0u : 0u) | ((w & 0x7f800000u) == 0x7f800000u ? 0x7fc00000u : 0u); }

__device__ inline float4v product(const Operand &a, const Operand &b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, c, 0, 0, 0); }
__device__ inline float16v product(const Operand &a, const Operand &b, float16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.b, b.b, c, 0, 0, 0); }

// A wave's NQ tiles of M rows
template <int D, int M, int NQ>
struct Wave {
    typedef Rows<D, M> R;
    typedef std::conditional_t<M == 16, float4v, float16v> Sums;
    static constexpr int kGroups = 64 / M, kSums = M / kGroups, kSteps = D / (8 * kGroups), kTiles = D / M, kKeys = 8 * kGroups;    // kSums: of a lane in a tile; kKeys: of an operand of values
    Operand q[NQ][kSteps];
    Sums o[kTiles][NQ];
    float top[NQ], sum[NQ];
    int lane, g, end[NQ];           // keys that the lane's rows see

    // The rows' queries on their way; take() waits for them, and for everything that was asked for since.
    __device__ void load(const Cut &w, const Sequence &s, int head, int row0, int rows, int lane_)
    {
        lane = lane_;
        g = lane / M;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int row = row0 + M * n + lane % M, r = min(row, rows - 1), i = r / w.group;
            top[n] = kNone;
            sum[n] = 0.0f;
            end[n] = row < rows ? visible(w.a, s, i) : 0;
            const uint16_t *const from = w.a.q + (long long)(s.q0 + i) * w.a.q_stride + (head * w.group + r - i * w.group) * D + 8 * g;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) q[n][k].u = *reinterpret_cast<const uint4 *>(from + 8 * kGroups * k);
        }
    }
    __device__ void take(const Cut &w)
    {
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) q[n][k].w[j] ^= w.flip;
        if (__builtin_expect(w.zero, 0))
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int k = 0; k < kSteps; ++k)
#pragma unroll
                    for (int j = 0; j < 4; ++j) q[n][k].w[j] = none_of(q[n][k].w[j]);
#pragma unroll
        for (int c = 0; c < kTiles; ++c)
#pragma unroll
            for (int n = 0; n < NQ; ++n) o[c][n] = Sums{};
    }
    // Scores of NK tiles of M keys at `keys` (LDS).
    template <int NK>
    __device__ void scores(const char *keys, Sums (&x)[NK][NQ]) const
    {
        const int row = lane % M;
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int m = 0; m < NK; ++m) {
                Operand a;
                a.u = *reinterpret_cast<const uint4 *>(keys + (row * R::kBytes + R::key_piece(row, kGroups * k + g) * 16) + M * m * R::kBytes);
#pragma unroll
                for (int n = 0; n < NQ; ++n) x[m][n] = product(a, q[n][k], k == 0 ? Sums{} : x[m][n]);
            }
    }
    // Unseen keys of NK tiles from number t on.
    template <int NK>
    __device__ void hide(Sums (&x)[NK][NQ], int t) const
    {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int seen = end[n] - t - 4 * g;
#pragma unroll
            for (int m = 0; m < NK; ++m)
#pragma unroll
                for (int i = 0; i < kSums; ++i) x[m][n][i] = M * m + 4 * kGroups * (i / 4) + i % 4 < seen ? x[m][n][i] : -INFINITY;
        }
    }
    // The largest scores of the rows.
    template <int NK>
    __device__ static void largest(const Sums (&x)[NK][NQ], float (&top)[NQ])
    {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float m = fmaxf(x[0][n][0], x[0][n][1]);
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
                for (int i = k == 0 ? 2 : 0; i < kSums; i += 2) m = fmaxf(fmaxf(m, x[k][n][i]), x[k][n][i + 1]);
            if (M == 16) {
                const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
                m = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
            }
            const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
            top[n] = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
        }
    }
    // ... and the maxima raised to them where that is called for.  Of every row for itself: its result does not depend on the wave's other rows.
    __device__ void raise(const float (&m)[NQ], const bool (&higher)[NQ], float scale2)
    {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const float next = higher[n] ? fmaxf(top[n], m[n]) : top[n], f = __builtin_amdgcn_exp2f((top[n] - next) * scale2);
            top[n] = next;
            sum[n] *= f;
#pragma unroll
            for (int c = 0; c < kTiles; ++c)
#pragma unroll
                for (int i = 0; i < kSums; ++i) o[c][n][i] *= f;
        }
    }
    // Where scores exceed a maximum by kSlack.
    template <int NK>
    __device__ void raise_to(const Sums (&x)[NK][NQ], float scale2)
    {
        float m[NQ];
        bool higher[NQ], any = false;
        largest(x, m);
#pragma unroll
        for (int n = 0; n < NQ; ++n) any |= higher[n] = (m[n] - top[n]) * scale2 > kSlack;
        if (__builtin_amdgcn_ballot_w64(any)) raise(m, higher, scale2);
    }
    // Where a row's weights of a step, of which each of its lanes has a sum, are too large, or its maximum is far out; whether there is such a row.
    template <int NK>
    __device__ bool raise_by(const float (&s)[NQ], const Sums (&x)[NK][NQ], float scale2)
    {
        bool any = false, higher_here[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) any |= higher_here[n] = !(fmaxf(s[n], fabsf(top[n] * scale2)) <= kMostWeights);       // (a sum that is no number stays one without this)
        if (!__builtin_amdgcn_ballot_w64(any)) return false;
        float m[NQ];
        bool higher[NQ];
        largest(x, m);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            uint32_t mine = higher_here[n];
            if (M == 16) {
                const auto r = __builtin_amdgcn_permlane16_swap(mine, mine, false, false);
                mine = r[0] | r[1];
            }
            const auto r = __builtin_amdgcn_permlane32_swap(mine, mine, false, false);
            higher[n] = (r[0] | r[1]) != 0;
        }
        raise(m, higher, scale2);
        return true;
    }
    // Weights of NK tiles of keys, as operands, and the lane's sums of them: without rows that are far out, and with any.
    template <int NK>
    __device__ void weights(const Sums (&x)[NK][NQ], float scale2, Operand (&p)[NK * M / kKeys][NQ], float (&s)[NQ]) const
    {
        float off[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) off[n] = top[n] * scale2;
        weights(x, scale2, off, p, s);
    }
    template <int NK>
    __device__ void weights_of_any(Sums (&x)[NK][NQ], float scale2, Operand (&p)[NK * M / kKeys][NQ], float (&s)[NQ]) const
    {
        // (a row that has seen nothing has weights of 0 from any finite `off`)
        float off[NQ];
        bool far[NQ], any = false;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            off[n] = fmaxf(top[n] * scale2, kNone);
            any |= far[n] = fabsf(off[n]) > kMostWeights && top[n] > kNone;
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(any) != 0, 0))
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const float from = far[n] ? top[n] : 0.0f;
                off[n] = far[n] ? 0.0f : off[n];
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int i = 0; i < kSums; ++i) x[k][n][i] -= from;
            }
        weights(x, scale2, off, p, s);
    }
    template <int NK>
    __device__ static void weights(const Sums (&x)[NK][NQ], float scale2, const float (&off)[NQ], Operand (&p)[NK * M / kKeys][NQ], float (&s)[NQ])
    {
        bf16x2 one;
        one[0] = one[1] = (__bf16)1.0f;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            s[n] = 0.0f;
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
                for (int i = 0; i < kSums; i += 2) {
                    const float a = __builtin_amdgcn_exp2f(fmaf(x[k][n][i], scale2, -off[n])), b = __builtin_amdgcn_exp2f(fmaf(x[k][n][i + 1], scale2, -off[n]));
                    const uint32_t both = pack_bf16x2(a, b);
                    p[(k * kSums + i) / 8][n].w[(k * kSums + i) % 8 / 2] = both;
                    s[n] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, both), one, s[n], false);
                }
        }
    }
    // The values of an operand's keys at `values` (LDS).
    __device__ void add(const char *values, const Operand (&p)[NQ])
    {
        const int i = lane & 15, row = 4 * g + (i >> 2);
#pragma unroll
        for (int c = 0; c < kTiles; ++c) {
            const char *const at = values + row * R::kBytes + R::value_piece(row, M / 8 * c + (M == 32 ? 2 * (lane >> 4 & 1) : 0) + (i >> 1 & 1)) * 16 + 8 * (i & 1);
            Operand a;
#pragma unroll
            for (int j = 0; j < 2; ++j)
                a.s[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v *)(const_cast<char *>(at) + 4 * kGroups * j * R::kBytes));
#pragma unroll
            for (int n = 0; n < NQ; ++n) o[c][n] = product(a, p[n], o[c][n]);
        }
    }
    // A value that is no number touches only the rows that see it: where `keys` rows of values have one and some rows of the wave do not see all of those keys, it is added to the rows that
    // do, here, before it is taken out of LDS: a weight is above 0, though exp2 of a far score is not, so an infinity stays one.  (In steps that all rows see the product has it: of a weight of 0, NaN.)
    __device__ void add_no_numbers(const char *values, int t, int keys)
    {
        for (int key = 0; key < keys; ++key)
#pragma unroll
            for (int c = 0; c < kTiles; ++c)
#pragma unroll
                for (int f = 0; f < kSums; f += 4) {
                    const int channel = M * c + kGroups * f + 4 * g;            // and the three behind it
                    const uint2 v = *reinterpret_cast<const uint2 *>(values + key * R::kBytes + R::value_piece(key, channel / 8) * 16 + 2 * (channel & 4));
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t bits = (i & 2 ? v.y : v.x) >> 16 * (i & 1) << 16;
                        if ((bits & 0x7f800000u) == 0x7f800000u)
#pragma unroll
                            for (int n = 0; n < NQ; ++n)
                                if (t + key < end[n]) o[c][n][f + i] += __uint_as_float(bits);
                    }
                }
    }
    // A row's parts of the lanes that have it.
    __device__ float total(int n) const
    {
        float s = sum[n];
        if (M == 16) {
            const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(s), __float_as_uint(s), false, false);
            s = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        }
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(s), __float_as_uint(s), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
};

// Whether 16 bytes have a bf16 infinity or NaN in them; the same without those.
__device__ inline bool no_numbers(const uint4 &v)
{
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
        bad |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
    }
    return bad;
}
__device__ inline uint32_t numbers_of(uint32_t w) { return w & ((w & 0x7f80u) == 0x7f80u ? 0xffff0000u : 0xffffffffu) & ((w & 0x7f800000u) == 0x7f800000u ? 0x0000ffffu : 0xffffffffu); }
// Pieces first, first + step, ... of `bytes` at `values`: whether there is one with no numbers, and taking those out.
__device__ inline bool find_no_numbers(const char *values, int bytes, int first, int step)
{
    bool bad = false;
    for (int at = 16 * first; at < bytes; at += 16 * step) bad |= no_numbers(*reinterpret_cast<const uint4 *>(values + at));
    return bad;
}
__device__ inline void take_out_no_numbers(char *values, int bytes, int first, int step)
{
    for (int at = 16 * first; at < bytes; at += 16 * step) {
        uint4 &v = *reinterpret_cast<uint4 *>(values + at);
        if (no_numbers(v)) v = make_uint4(numbers_of(v.x), numbers_of(v.y), numbers_of(v.z), numbers_of(v.w));
    }
}

// ---- from memory into LDS
__device__ inline uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)p; }
// One transfer: rows first .. first + kPerTransfer - 1 of those at `from` (rows past `most` are read as that one), to `lds` + their place.  ONCE: of rows that nobody else reads, past the caches.
template <class R, bool KEYS, bool ONCE>
__device__ inline void transfer(const uint16_t *from, long long stride, int first, int most, uint32_t lds, int lane)
{
    const int row = first + lane / R::kPieces, c = lane % R::kPieces;
    const int piece = KEYS ? R::key_piece(row, c) : R::value_piece(row, c);
    const uint32_t at = (uint32_t)(min(row, most) * (int)stride * 2 + piece * 16);
    if (ONCE) dma16_once(at, from, lds + first * R::kBytes);
    else dma16(at, from, lds + first * R::kBytes);
}

template <int D>
constexpr int kPartial = D + 2;
__device__ inline size_t partial_row(const Cut &w, int b, int head, int row, int split)
{
    return (((size_t)b * w.a.kv_heads + head) * ((size_t)w.a.max_q * w.group) + row) * w.splits + split;
}

// The order in which a step's instructions are issued: vector instructions and LDS reads between the products, evenly (13740 rows on as many keys, 16 heads x 64: 809 us for 826 in the compiler's
// order; 8192 on 8192, 16 x 128: 485 and 521).
template <int D>
__device__ inline void pace_scores()
{
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);              // reads of keys ahead; then a product, vector instructions, a read
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, D == 128 ? 5 : 8, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
}
template <int D>
__device__ inline void pace_values()
{
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
}

// ---- many rows: a wave has 32 of its own, the four waves of a block go through the same keys, 64 a step, two tiles of each in LDS.  Products of 32 x 32 x 16: a lane's registers hold a tile and
// the scores of the next one, for which 16 x 16 x 32, faster out of registers alone, leave no room (8192 rows on 8192 keys, 16 heads x 128: 516 us for 493).  Bound by the board's power where sequences are
// long: 11003 tokens, 32 heads on 8 x 128, 877 to 902 us by the board, 1.10 to 1.13 PFLOP/s at 1.6 GHz, with the matrix cores busy in 0.65 of the cycles, and 651 us on zeros; with 64 channels by vector
// instructions as well (97 for 16 products a step: 13740 rows on as many keys, 16 heads, 798 to 816 us, 0.95 to 0.97 PFLOP/s).  A block costs some 8 us besides its steps.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void attention_own_rows_kernel(Cut w)
{
    typedef Rows<D, 32> R;
    constexpr int kKeys = 64, kTile = kKeys * R::kBytes, kEach = kKeys / R::kPerTransfer / 4;
    __shared__ __align__(16) char area[4 * kTile];          // two tiles of keys, two of values
    char *const keys = area, *const values = area + 2 * kTile;
    const Attention &a = w.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Heads first, then tiles from the last one on, where rows see most, then sequences, parts of the keys last: blocks that run together have keys in common (those of a head on one of the eight
    // dies, where heads are a multiple of eight), a sequence's longest blocks begin first, and a part that has less to do than another is on all dies alike (a prompt of 16384 tokens in two parts,
    // 16 heads on 4: 613 us for 884 with parts side by side)
    const int head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, place = rest % w.tiles, b = rest / w.tiles % a.seqs, split = rest / w.tiles / a.seqs;
    const Sequence seq = sequence_of(a, b);
    const int rows = seq.n * w.group, tile = (rows + 127) / 128 - 1 - place;
    if (tile < 0) return;
    const int row0 = tile * 128, row = row0 + 32 * wave + (lane & 31), rows_end = min(rows, row0 + 128);
    const int last = visible(a, seq, (rows_end - 1) / w.group), full = visible(a, seq, row0 / w.group);        // keys that some row of the block sees, and that all see
    const int t0 = split * w.chunk, stop = min(last, t0 + w.chunk), steps = (stop - t0 + kKeys - 1) / kKeys;
    if (split > 0 && t0 >= last) return;
    Wave<D, 32, 1> r;
    r.load(w, seq, head, row0 + 32 * wave, rows, lane);
    const uint16_t *const k = a.k + (long long)(seq.k0 + t0) * a.k_stride + head * D, *const v = a.v + (long long)(seq.k0 + t0) * a.v_stride + head * D;
    // A lane's place in this wave's transfers of a tile: the keys' pieces change with the row, the values' do not from transfer to transfer
    uint32_t from_key[kEach], from_value;
    const int row_of_lane = lane / R::kPieces, piece = lane % R::kPieces, first = wave * kEach * R::kPerTransfer;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int at = first + i * R::kPerTransfer + row_of_lane;
        from_key[i] = (uint32_t)(at * (int)a.k_stride * 2 + R::key_piece(at, piece) * 16);
    }
    from_value = (uint32_t)((first + row_of_lane) * (int)a.v_stride * 2 + R::value_piece(first + row_of_lane, piece) * 16);
    const uint32_t lds = lds_address(area) + first * R::kBytes;
    auto bring_keys = [&](int step, int buffer) {
        const uint16_t *const from = k + (long long)step * kKeys * a.k_stride;
        const uint32_t to = lds + buffer * kTile;
        if (t0 + (step + 1) * kKeys <= last) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) dma16(from_key[i], from, to + i * R::kPerTransfer * R::kBytes);
        } else
#pragma unroll
            for (int i = 0; i < kEach; ++i) transfer<R, true, false>(from, a.k_stride, first + i * R::kPerTransfer, last - 1 - t0 - step * kKeys, lds_address(keys) + buffer * kTile, lane);
    };
    auto bring_values = [&](int step, int buffer) {
        const uint16_t *const from = v + (long long)step * kKeys * a.v_stride;
        const uint32_t to = lds + (2 + buffer) * kTile;
        if (t0 + (step + 1) * kKeys <= last) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) dma16(from_value, from + (long long)i * R::kPerTransfer * a.v_stride, to + i * R::kPerTransfer * R::kBytes);
        } else
#pragma unroll
            for (int i = 0; i < kEach; ++i) transfer<R, false, false>(from, a.v_stride, first + i * R::kPerTransfer, last - 1 - t0 - step * kKeys, lds_address(values) + buffer * kTile, lane);
    };
    auto arrived = [] {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    if (steps > 0) {        // two tiles of keys at once (eight chunks of 61 rows, 71 us for 73; 20 frames of 1374 tokens, 16 heads x 64, 126 for 127)
        bring_keys(0, 0);
        bring_values(0, 0);
        if (steps > 1) bring_keys(1, 1);
    }
    r.take(w);
    if (steps > 0) {
        // While a step's weights are made the next one's scores are multiplied: keys are a step ahead of values
        float16v x[2][1], y[2][1];
        Operand p[4][1];
        arrived();
        r.scores(keys, x);
        float s[1];
        __syncthreads();
        // Steps that every row of the block sees, two at a time; behind each of them there is another
        const int plain = min(max(full - t0, 0) / kKeys, steps - 1) & ~1;
        int step = 0;
        auto both = [&](auto parity, float16v(&x)[2][1], float16v(&y)[2][1]) {
            constexpr int kHere = decltype(parity)::value, kNext = kHere ^ 1;
            if (step + 2 < steps) bring_keys(step + 2, kHere);
            bring_values(step + 1, kNext);
            r.scores(keys + kNext * kTile, y);
            r.weights(x, w.scale2, p, s);
            pace_scores<D>();
            if (r.raise_by(s, x, w.scale2)) r.weights_of_any(x, w.scale2, p, s);
            r.sum[0] += s[0];
#pragma unroll
            for (int i = 0; i < 4; ++i) r.add(values + kHere * kTile + 16 * i * R::kBytes, p[i]);
            pace_values<D>();
            ++step;
            arrived();
        };
        while (step < plain) {
            both(std::integral_constant<int, 0>(), x, y);
            both(std::integral_constant<int, 1>(), y, x);
        }
        for (; step < steps; ++step) {
            const int here = step & 1;
            const bool more = step + 1 < steps;
            if (step + 2 < steps) bring_keys(step + 2, here);
            if (more) {
                bring_values(step + 1, here ^ 1);
                r.scores(keys + (here ^ 1) * kTile, y);
            }
            const int t = t0 + step * kKeys;
            char *const mine = values + here * kTile;
            bool bad = false;
            if (t + kKeys > full) {
                r.hide(x, t);
                bad = __syncthreads_or(find_no_numbers(mine, kTile, threadIdx.x, 256));
            }
            r.raise_to(x, w.scale2);
            r.weights_of_any(x, w.scale2, p, s);
            r.sum[0] += s[0];
            if (bad) {
                r.add_no_numbers(mine, t, kKeys);
                __syncthreads();
                take_out_no_numbers(mine, kTile, threadIdx.x, 256);
                __syncthreads();
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) r.add(mine + 16 * i * R::kBytes, p[i]);
            if (more) {
                x[0][0] = y[0][0];
                x[1][0] = y[1][0];
            }
            arrived();
        }
    }
    const float total = r.total(0);
    if (w.splits == 1) {
        const float f = share_of(total, r.end[0]);
        const int i = row / w.group;
        uint16_t *const to = a.out + ((long long)(seq.q0 + i) * a.q_heads + head * w.group + row - i * w.group) * D;
        // Of sixteen channels, of which the two lanes of a row have fours in turn, each comes to have eight neighbouring ones
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
                uint32_t word[4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const auto s = __builtin_amdgcn_permlane32_swap(pack_bf16x2(r.o[c][0][e + 2 * j] * f, r.o[c][0][e + 2 * j + 1] * f),
                                                                    pack_bf16x2(r.o[c][0][e + 4 + 2 * j] * f, r.o[c][0][e + 4 + 2 * j + 1] * f), false, false);
                    word[j] = s[0];
                    word[2 + j] = s[1];
                }
                if (row < rows) *reinterpret_cast<uint4 *>(to + 32 * c + 2 * e + 8 * r.g) = make_uint4(word[0], word[1], word[2], word[3]);
            }
    } else if (row < rows) {
        float *const to = w.partials + partial_row(w, b, head, row, split) * kPartial<D>;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int e = 0; e < 16; e += 2) *reinterpret_cast<float2 *>(to + 32 * c + 8 * (e / 4) + 4 * r.g + e % 4) = make_float2(r.o[c][0][e], r.o[c][0][e + 1]);
        if (r.g == 0) *reinterpret_cast<float2 *>(to + D) = make_float2(r.top[0], total);
    }
}

// ---- few rows (32 at most): the waves of a block share them and go through keys of their own, 32 at a time, brought into LDS by each for itself.  Products of 16 x 16 x 32, of whose rows fewer are
// nobody's.  Bound by memory: 48 rows on up to 8192 keys, 32 heads on 8 x 128, 148 us, 5.8 TB/s; a block alone on a CU brings in 52 GB/s (one row on 601 keys: 7.4 us)
template <int D, int NQ, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 4 ? 2 : 1) void attention_few_rows_kernel(Cut w)
{
    typedef Rows<D, 16> R;
    constexpr int kKeys = 32, kTile = kKeys * R::kBytes, kEach = kKeys / R::kPerTransfer;
    extern __shared__ __align__(16) char few_area[];        // a tile of keys and one of values for every wave
    __shared__ float tops[WAVES][16 * NQ], totals[WAVES][16 * NQ];
    const Attention &a = w.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, split = rest % w.splits, b = rest / w.splits;
    const Sequence seq = sequence_of(a, b);
    const int rows = seq.n * w.group;
    if (rows == 0) return;
    const int last = visible(a, seq, seq.n - 1), full = visible(a, seq, 0), t0 = split * w.chunk, stop = min(last, t0 + w.chunk);
    if (split > 0 && t0 >= last) return;
    Wave<D, 16, NQ> r;
    const uint16_t *const k = a.k + (long long)seq.k0 * a.k_stride + head * D, *const v = a.v + (long long)seq.k0 * a.v_stride + head * D;
    char *const keys = few_area + wave * 2 * kTile, *const values = keys + kTile;
    auto bring_keys = [&](int t) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) transfer<R, true, true>(k + (long long)t * a.k_stride, a.k_stride, i * R::kPerTransfer, last - 1 - t, lds_address(keys), lane);
    };
    auto bring_values = [&](int t) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) transfer<R, false, true>(v + (long long)t * a.v_stride, a.v_stride, i * R::kPerTransfer, last - 1 - t, lds_address(values), lane);
    };
    r.load(w, seq, head, 0, rows, lane);
    int t = t0 + kKeys * wave;
    if (t < stop) {
        bring_keys(t);
        bring_values(t);
    }
    r.take(w);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");        // the queries and the first tile: from here on only transfers are counted
    for (; t < stop; t += WAVES * kKeys) {
        const bool more = t + WAVES * kKeys < stop;
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kEach) : "memory");        // the keys; the values are on their way
        lanes_exchange_fence();
        float4v x[2][NQ];
        Operand p[1][NQ];
        float s[NQ];
        r.scores(keys, x);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) bring_keys(t + WAVES * kKeys);
        const bool masked = t + kKeys > full;
        if (masked) r.hide(x, t);
        r.raise_to(x, w.scale2);
        r.weights_of_any(x, w.scale2, p, s);
#pragma unroll
        for (int n = 0; n < NQ; ++n) r.sum[n] += s[n];
        if (more) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kEach) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lanes_exchange_fence();
        if (masked && __builtin_amdgcn_ballot_w64(find_no_numbers(values, kTile, lane, 64))) {
            r.add_no_numbers(values, t, kKeys);
            lanes_exchange_fence();
            take_out_no_numbers(values, kTile, lane, 64);
            lanes_exchange_fence();
        }
        r.add(values, p[0]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) bring_values(t + WAVES * kKeys);
    }
    // The waves' sums, in the LDS that held their tiles: rows of D floats, their pieces of four in an order by the row
    constexpr int kFours = D / 4;
    float *const mine = reinterpret_cast<float *>(keys);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int here = 16 * n + (lane & 15);
        const float total = r.total(n);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) *reinterpret_cast<float4 *>(mine + here * D + ((4 * c + r.g) ^ (here & (kFours - 1))) * 4) = make_float4(r.o[c][n][0], r.o[c][n][1], r.o[c][n][2], r.o[c][n][3]);
        if (r.g == 0) {
            tops[wave][here] = r.top[n];
            totals[wave][here] = total;
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * kFours; i += 64 * WAVES) {
        const int row = i / kFours, c = i % kFours;
        float top = kNone, all = 0.0f;
#pragma unroll
        for (int n = 0; n < WAVES; ++n) top = fmaxf(top, tops[n][row]);
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int n = 0; n < WAVES; ++n) {
            const float f = __builtin_amdgcn_exp2f((tops[n][row] - top) * w.scale2);
            const float4 y = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(few_area + n * 2 * kTile) + row * D + (c ^ (row & (kFours - 1))) * 4);
            all = fmaf(f, totals[n][row], all);
            x = make_float4(fmaf(f, y.x, x.x), fmaf(f, y.y, x.y), fmaf(f, y.z, x.z), fmaf(f, y.w, x.w));
        }
        if (w.splits == 1) {
            const int at = row / w.group;
            const float f = share_of(all, visible(a, seq, at));
            *reinterpret_cast<uint2 *>(a.out + ((long long)(seq.q0 + at) * a.q_heads + head * w.group + row - at * w.group) * D + 4 * c) =
                make_uint2(pack_bf16x2(x.x * f, x.y * f), pack_bf16x2(x.z * f, x.w * f));
        } else {
            float *const to = w.partials + partial_row(w, b, head, row, split) * kPartial<D>;
            *reinterpret_cast<float2 *>(to + 4 * c) = make_float2(x.x, x.y);
            *reinterpret_cast<float2 *>(to + 4 * c + 2) = make_float2(x.z, x.w);
            if (c == 0) *reinterpret_cast<float2 *>(to + D) = make_float2(top, all);
        }
    }
}

// ---- the parts of a row put together: 16 lanes have a row.  Every lane finds the factors of some of the parts, which all need
template <int D>
__global__ __launch_bounds__(256) void attention_join_kernel(Cut w)
{
    constexpr int C = D / 16;
    __shared__ float factors[16][kAttentionMostParts];
    const Attention &a = w.a;
    const int lane = threadIdx.x & 15, first = lane * C, blocks = (a.max_q * w.group + 15) / 16;
    const int head = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads, b = rest / blocks, row = rest % blocks * 16 + (threadIdx.x >> 4);
    const Sequence seq = sequence_of(a, b);
    if (row >= seq.n * w.group) return;
    const int i = row / w.group, seen = visible(a, seq, i), used = (seen + w.chunk - 1) / w.chunk;
    const float *const from = w.partials + partial_row(w, b, head, row, 0) * kPartial<D>;
    float *const mine = factors[threadIdx.x >> 4];
    float top = kNone, total = 0.0f, x[C];
    for (int s = lane; s < used; s += 16) top = fmaxf(top, from[(size_t)s * kPartial<D> + D]);
    top = max_over_16_lanes(top);
    for (int s = lane; s < used; s += 16) {
        const float2 p = *reinterpret_cast<const float2 *>(from + (size_t)s * kPartial<D> + D);
        mine[s] = __builtin_amdgcn_exp2f((p.x - top) * w.scale2);
        total = fmaf(mine[s], p.y, total);
    }
    lanes_exchange_fence();
    total = dpp_add_step<0xB1>(total);
    total = dpp_add_step<0x4E>(total);
    total = dpp_add_step<0x141>(total);
    total = dpp_add_step<0x140>(total);
#pragma unroll
    for (int c = 0; c < C; ++c) x[c] = 0.0f;
#pragma unroll 4
    for (int s = 0; s < used; ++s) {
        const float *const p = from + (size_t)s * kPartial<D> + first;
        const float f = mine[s];
#pragma unroll
        for (int c = 0; c < C; c += 2) {
            const float2 v = *reinterpret_cast<const float2 *>(p + c);
            x[c] = fmaf(f, v.x, x[c]);
            x[c + 1] = fmaf(f, v.y, x[c + 1]);
        }
    }
    const float f = share_of(total, seen);
    uint32_t *const to = reinterpret_cast<uint32_t *>(a.out + ((long long)(seq.q0 + i) * a.q_heads + head * w.group + row - i * w.group) * D + first);
#pragma unroll
    for (int c = 0; c < C; c += 2) to[c / 2] = pack_bf16x2(x[c] * f, x[c + 1] * f);
}

#define FEW(d, nq, waves) {reinterpret_cast<const void *>(attention_few_rows_kernel<d, nq, waves>), waves * 128 * d}
const LdsKernel lds_kernels_list[] = {FEW(64, 1, 4), FEW(64, 1, 8), FEW(64, 2, 4), FEW(64, 2, 8), FEW(128, 1, 4), FEW(128, 1, 8), FEW(128, 2, 4), FEW(128, 2, 8)};
#undef FEW
const LdsKernels lds_kernels(lds_kernels_list);

template <int D>
hipError_t launch(const Attention &a, hipStream_t stream)
{
    const int group = a.q_heads / a.kv_heads;
    const AttentionPlan p = attention_plan(a.seqs, a.max_q, a.max_kv, a.q_heads, a.kv_heads, D, a.causal);
    const float scale2 = a.scale == 0.0f ? 1.0f : __builtin_fabsf(a.scale) * kLog2e;
    const Cut w{a, group, p.chunk, p.splits, p.tiles, scale2, a.scale < 0.0f ? 0x80008000u : 0u, a.scale == 0.0f,
                static_cast<float *>(a.workspace)};
    const dim3 grid((unsigned)a.seqs * a.kv_heads * p.tiles * p.splits);
    hipError_t e = p.few ? prepare_device() : hipSuccess;
    if (e != hipSuccess) return e;
    const bool one = (long long)a.max_q * group <= 16;
    if (p.few && p.waves == 8) (one ? attention_few_rows_kernel<D, 1, 8> : attention_few_rows_kernel<D, 2, 8>)<<<grid, 512, 8 * 128 * D, stream>>>(w);
    else if (p.few) (one ? attention_few_rows_kernel<D, 1, 4> : attention_few_rows_kernel<D, 2, 4>)<<<grid, 256, 4 * 128 * D, stream>>>(w);
    else attention_own_rows_kernel<D><<<grid, 256, 0, stream>>>(w);
    e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    attention_join_kernel<D><<<dim3((unsigned)a.seqs * a.kv_heads * ((a.max_q * group + 15) / 16)), 256, 0, stream>>>(w);
    return hipGetLastError();
}

}  // namespace

hipError_t run_attention(const Attention &a, int d, hipStream_t stream) { return d == 64 ? launch<64>(a, stream) : launch<128>(a, stream); }

}  // namespace qvggt

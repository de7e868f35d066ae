// Attention over the 4-bit key/value cache: qvggt_kv4_attention.
//
//     o = softmax_j(scale <q, k_j>) v_j,   k_j = step (code_j H) s,  v_j likewise:   <q, k_j> = step <(s q) H, code_j>,   o = s ((sum_j p_j step_j code_j) H)
//
// so queries are turned once, products are taken with the codes themselves, a token's step is a factor of its score or its weight, and the sum is turned back at the end.
//
// The codes go to the matrix cores as fp16 numbers without a conversion: u = code + 8 in the low four bits of a half word is the subnormal u 2^-24, one nibble
// up it is 16 u 2^-24, both exact (the instruction does not flush them), so a word of 8 codes is four operands after one shift and four ands.  The 16 of the odd channels is taken
// out of the queries in the one product and out of the sum in the other, and the 8 that every code is too large by comes off in the accumulator that the first product starts from
// and, in the second, with the sum of the weights that one more instruction on eights makes.  Queries are fp16 with a power of two common to a wave, weights fp16 scaled so
// that they reach down to 2^-31 of the largest: 11 bits, against 8 of a bf16 that the result is rounded to.
//
// A wave takes 32 tokens a step: scores of 32 tokens x 16 rows (keys x queries), exp2, weights, sums (values x weights) -- the accumulators of the first product have, lane by lane, the
// tokens that the second product's operand needs, so nothing moves between lanes.  Rows are the query tokens of a sequence times the query heads that share a key head.
#include "kv4.h"

namespace qvggt {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __fp16 half2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));

union Operand {                 // eight fp16 numbers of a lane
    uint32_t w[4];
    half8 h;
};

__device__ inline float4v mfma(const Operand &a, const Operand &b, float4v c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, b.h, c, 0, 0, 0); }

constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNone = -1e30f;                 // running maximum of a row that has seen nothing
constexpr float kSlack = 8.0f;                  // weights may pass 1 by this many powers of two before sums are scaled down
constexpr float kTop = 128.0f;                  // weight of a score at the running maximum with the largest step: 2^15 with the slack, under fp16's 65504

struct Work {
    Kv4Attention a;
    int group;                  // query heads of a key head
    int chunk, splits;          // keys of a block of waves, and how many of those there may be
};

// what a block knows about its sequence
struct Sequence {
    int start, n, len;
};
__device__ inline Sequence sequence_of(const Kv4Attention &a, int b)
{
    Sequence s;
    s.start = min(max(a.starts[b], 0), a.T);
    s.n = min(min(max(a.starts[b + 1] - s.start, 0), a.max_q), a.T - s.start);
    s.len = min(max(a.lens[b], 0), a.max_kv);
    return s;
}
// keys that a query token sees
__device__ inline int visible(const Kv4Attention &a, const Sequence &s, int token) { return a.causal ? min(max(s.len - s.n + token + 1, 0), s.len) : s.len; }

// one row of 16 lanes' worth of a sum, turned back and written
template <int D>
__device__ inline void finish_row(const Kv4Attention &a, int group, const Sequence &s, int head, int row, float (&x)[D / 16], float factor, int lane)
{
    constexpr int C = D / 16;
    const int first = (lane & 15) * C;
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] *= factor;
    row_butterflies<C>(x, lane);
    sign_channels<C>(a.signs, first, x);
    uint16_t *to = a.out + ((size_t)(s.start + row / group) * a.q_heads + head * group + row % group) * D + first;
#pragma unroll
    for (int i = 0; i < C / 4; ++i) reinterpret_cast<uint2 *>(to)[i] = make_uint2(pack_bf16x2(x[4 * i], x[4 * i + 1]), pack_bf16x2(x[4 * i + 2], x[4 * i + 3]));
}

// floats of a row of one split's partial sums: D sums, the maximum, the sum of weights
template <int D>
constexpr int kPartial = D + 2;
__device__ inline size_t partial_row(const Kv4Attention &a, int group, int splits, int b, int head, int row, int split)
{
    return (((size_t)b * a.pages.heads + head) * ((size_t)a.max_q * group) + row) * splits + split;
}

// What a wave holds of 32 tokens: words of keys and values and the steps, as they lie in the pages.
template <int D>
struct Step {
    uint32_t k[2][D / 32], v[2][D / 32];
    uint32_t s[2][4];
};

// waves that a SIMD's registers hold: as many as leave none of them in scratch memory
template <int D, int NT>
constexpr int kWavesPerSimd = NT == 4 ? 1 : NT == 2 ? 2 : D == 64 ? 4 : 3;

// Waves of a block share rows and take steps of 32 keys in turn (SHARE, up to 16 NT rows: few rows, many keys), or have 16 NT rows each.
template <int D, int NT, bool SHARE>
__global__ __launch_bounds__(256, (kWavesPerSimd<D, NT>)) void kv4_attention_kernel(Work work)
{
    using L = Kv4Layout<D>;
    constexpr int C = D / 16, W = L::kWords, S = D / 32;
    constexpr int kPad = D + 4;                             // floats of a row in LDS
    constexpr int kStride = SHARE ? 128 : 32;               // keys from a wave's step to its next
    __shared__ __align__(16) float area[4][16 * kPad];
    __shared__ float row_max[4][16], row_sum[4][16];
    const Kv4Attention &a = work.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const int split = blockIdx.x % work.splits, tile = blockIdx.x / work.splits;
    const int head = blockIdx.y, b = blockIdx.z, group = work.group;
    const Sequence seq = sequence_of(a, b);
    const int rows = seq.n * group, row0 = SHARE ? tile * 16 * NT : (tile * 4 + wave) * 16 * NT;
    if (SHARE ? row0 >= rows : tile * 64 * NT >= rows) return;
    float *const mine = area[wave];

    // ---- keys of this block
    const int rows_here = min(max(rows - row0, 0), 16 * NT);
    const int last = rows_here > 0 ? visible(a, seq, (row0 + rows_here - 1) / group) : 0;       // keys that some row of the wave's sees
    const int full = rows_here > 0 ? visible(a, seq, row0 / group) : 0;                         // keys that all of them see
    const int begin = split * work.chunk, stop = min(last, begin + work.chunk);
    if (SHARE && begin >= last && split > 0) return;            // nobody reads what this split would have left (rows without keys at all: the first split's)

    // The way of a step: its blocks' pages two steps ahead (scalar loads), its bytes into the registers of the step before as soon as those are taken apart.  Blocks behind the end
    // are taken as the last one.
    const int page_shift = a.pages.page_shift, page_mask = (1 << page_shift) - 1, last_block = max(last - 1, 0) / 16;
    const auto *const table = reinterpret_cast<const __attribute__((address_space(4))) int32_t *>(reinterpret_cast<uintptr_t>(a.table + (size_t)b * a.table_width));
    const size_t part_bytes = (size_t)(D + 4) << page_shift;
    const uint8_t *const head_base = a.pages.base + head * part_bytes;
    auto find = [&](int t0, int (&page)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) page[h] = table[min(t0 / 16 + h, last_block) * 16 >> page_shift];
    };
    const uint8_t *part[2];                     // the next step's blocks: head parts of pages, and tokens in them
    int at[2];
    auto locate = [&](int t0, const int (&page)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            at[h] = min(t0 / 16 + h, last_block) * 16 & page_mask;
            part[h] = head_base + (size_t)min(max(page[h], 0), a.pages.num_pages - 1) * (a.pages.heads * part_bytes);
        }
    };
    auto words = [&](const uint8_t *from, uint32_t (&w)[W]) {
        if constexpr (W == 4) {
            const uint4 v = *reinterpret_cast<const uint4 *>(from);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2 *>(from);
            w[0] = v.x; w[1] = v.y;
        }
    };
    const int key_of_lane = n16 * L::kRow + g * 4 * W, value_of_lane = lane * 4 * W;
    Step<D> x;
    auto fetch_keys = [&](int h) { words(part[h] + L::keys(at[h]) + key_of_lane, x.k[h]); };
    auto fetch_values = [&](int h) { words(part[h] + L::values(at[h], page_shift) + value_of_lane, x.v[h]); };
    auto fetch_steps = [&](int h) {
        const uint4 v = *reinterpret_cast<const uint4 *>(part[h] + L::steps(at[h], page_shift) + 16 * g);
        x.s[h][0] = v.x; x.s[h][1] = v.y; x.s[h][2] = v.z; x.s[h][3] = v.w;
    };
    int t0 = begin + (SHARE ? wave * 32 : 0), page[2] = {0, 0};
    if (t0 < stop) {
        find(t0, page);
        locate(t0, page);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            fetch_keys(h);
            fetch_steps(h);
            fetch_values(h);
        }
        find(t0 + kStride, page);
    }

    // ---- queries: four rows at a time to LDS, turned; then the lane's operands.  Lane (n, g) has channels g D / 4 .. of row n, as the keys' lanes have
    Operand q[NT][S];
    float base[NT];                     // what the first product starts from: -8 times the sum of the queries
    int end[NT];                        // keys that the lane's row sees
    float exponent[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int r = row0 + 16 * j + n16;
        end[j] = r < rows ? visible(a, seq, r / group) : 0;
        float *const turned = SHARE ? area[j & 3] : mine;          // shared rows: a quarter of them by every wave
#pragma unroll
        for (int k = 0; k < (SHARE ? 1 : 4); ++k) {
            const int r16 = SHARE ? 4 * wave + g : 4 * k + g, row = row0 + 16 * j + r16, first = n16 * C;
            float x[C];
#pragma unroll
            for (int i = 0; i < C; ++i) x[i] = 0.0f;
            if (row < rows) {
                const long long token = seq.start + row / group;
                const char *from = static_cast<const char *>(a.q) + (token * a.q_stride + (long long)(head * group + row % group) * D) * (a.q_f32 ? 4 : 2);
                load_channels<C>(from, a.q_f32, first, x);
                if (a.rope.table != nullptr) rotate_channels<C>(from, a.q_f32, first, a.rope, min(max(a.rope.positions[token], 0), a.rope.rows - 1), x);
                sign_channels<C>(a.signs, first, x);
            }
            row_butterflies<C>(x, lane);
            const float f = kv4_norm<D>() * a.scale * kLog2e;
#pragma unroll
            for (int i = 0; i < C; ++i) turned[r16 * kPad + first + i] = x[i] * f;
        }
        if constexpr (SHARE) __syncthreads();
        else lanes_exchange_fence();
        float x[D / 4], top = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 4; ++i) {
            x[i] = turned[n16 * kPad + g * (D / 4) + i];
            top = fmaxf(top, fabsf(x[i]));
        }
        if constexpr (!SHARE) lanes_exchange_fence();
        top = max_over_64_lanes(top);
        // 2^(13 - e) with 2^e <= top < 2^(e + 1): the largest query number of the tile in 2^13 .. 2^14, the others to an absolute error that is 2^-25 of a score unit at least.
        // Numbers over 2^17 (scores in the ten thousands at least: one key takes all the weight) become the largest fp16 and leave the other rows alone
        const int e = min(max((int)(__float_as_uint(top) >> 23), 20), 127 + 16);
        exponent[j] = (float)(e - 127 - 13);
        const float up = __uint_as_float((uint32_t)(127 + 13 - (e - 127)) << 23);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                y[i] = x[8 * s + i] * up;
                if (fabsf(y[i]) > 65504.0f) y[i] = copysignf(65504.0f, y[i]);
                if (i & 1) y[i] *= 0.0625f;
            }
            constexpr int order[8] = {0, 4, 1, 5, 2, 6, 3, 7};
#pragma unroll
            for (int i = 0; i < 8; ++i) q[j][s].h[i] = (_Float16)y[order[i]];
        }
    }
    float highest = exponent[0];
#pragma unroll
    for (int j = 1; j < NT; ++j) highest = fmaxf(highest, exponent[j]);
    const float unit = __builtin_amdgcn_exp2f(highest + 24.0f);     // of a product of a query number and a subnormal
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const _Float16 down = (_Float16)__builtin_amdgcn_exp2f(fmaxf(exponent[j] - highest, -40.0f));
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
    }

    float4v acc[NT][2 * W], ones[NT];
    float m[NT], l[NT];
    float reach = 0.0f, per = 0.0f;                             // power of two that no value's step so far is above; kTop / reach
    const float4v zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int c = 0; c < 2 * W; ++c) acc[j][c] = zero;
        ones[j] = zero;
        m[j] = kNone;
        l[j] = 0.0f;
    }
    Operand eights;
#pragma unroll
    for (int i = 0; i < 4; ++i) eights.w[i] = 0x00080008u;

    // 32 keys; edge: some row does not see all of them
    auto take = [&](auto edge) {
        constexpr bool kEdge = decltype(edge)::value;
        float ks[2][4], vs[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                ks[h][i] = __uint_as_float(x.s[h][i] << 16) * unit;
                vs[h][i] = __uint_as_float(x.s[h][i] & 0xffff0000u);
                if (kEdge && t0 + 16 * h + 4 * g + i >= last) vs[h][i] = 0.0f;             // behind the end lies whatever was there: no number, perhaps
            }
        locate(t0 + kStride, page);
        find(t0 + 2 * kStride, page);
        // scores, in powers of two above the running maximum
        float4v sc[NT][2];
        float t[NT][2][4], over = kNone, tops = 0.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            Operand k[S];
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const uint32_t w = x.k[h][s], u = w >> 8;
                k[s].w[0] = w & kLow; k[s].w[1] = w & kHigh; k[s].w[2] = u & kLow; k[s].w[3] = u & kHigh;
            }
            fetch_keys(h);
            fetch_steps(h);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                sc[j][h] = float4v{base[j], base[j], base[j], base[j]};
#pragma unroll
                for (int s = 0; s < S; ++s) sc[j][h] = mfma(k[s], q[j][s], sc[j][h]);
            }
        }
        auto above = [&](int j, int h, int i) {
            const float v = fmaf(sc[j][h][i], ks[h][i], -m[j]);
            return kEdge && t0 + 16 * h + 4 * g + i >= end[j] ? -INFINITY : v;
        };
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                tops = fmaxf(tops, vs[h][i]);
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    t[j][h][i] = above(j, h, i);
                    over = fmaxf(over, t[j][h][i]);
                }
            }
        if (__builtin_amdgcn_ballot_w64(over > kSlack || tops > reach)) {
            tops = max_over_64_lanes(tops);
            float shrink = 1.0f;
            if (tops > reach) {
                const float up = __uint_as_float(min((__float_as_uint(tops) & 0x7f800000u) + 0x00800000u, 0x7f000000u));
                shrink = reach / up;
                reach = up;
                per = kTop / up;
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                float top = m[j];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!kEdge || t0 + 16 * h + 4 * g + i < end[j]) top = fmaxf(top, sc[j][h][i] * ks[h][i]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float down = __builtin_amdgcn_exp2f(m[j] - top);
                m[j] = top;
                l[j] *= down;
                const float both = down * shrink;
#pragma unroll
                for (int i = 0; i < 4; ++i) ones[j][i] *= both;
#pragma unroll
                for (int c = 0; c < 2 * W; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[j][c][i] *= both;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) t[j][h][i] = above(j, h, i);
            }
        }
        // weights: tokens 0, 2 and 1, 3 of a group of four, as the bytes of a value's word come apart
        Operand p[NT];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float f[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = vs[h][i] * per;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f(t[j][h][i]);
                l[j] += (e[0] + e[1]) + (e[2] + e[3]);
                p[j].w[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(e[0] * f[0], e[2] * f[2]));
                p[j].w[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(e[1] * f[1], e[3] * f[3]));
            }
        }
#pragma unroll
        for (int w = 0; w < W; ++w) {
            Operand low, high;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t v = x.v[h][w], u = v >> 8;
                low.w[2 * h] = v & kLow; low.w[2 * h + 1] = u & kLow;
                high.w[2 * h] = v & kHigh; high.w[2 * h + 1] = u & kHigh;
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                acc[j][2 * w] = mfma(low, p[j], acc[j][2 * w]);
                acc[j][2 * w + 1] = mfma(high, p[j], acc[j][2 * w + 1]);
            }
        }
        fetch_values(0);
        fetch_values(1);
#pragma unroll
        for (int j = 0; j < NT; ++j) ones[j] = mfma(eights, p[j], ones[j]);
    };
    for (const int whole = min(full, stop) - 32; t0 <= whole; t0 += kStride) take(std::false_type());       // (one loop with both in it takes 70 registers more)
    for (; t0 < stop; t0 += kStride) take(std::true_type());

    // ---- sums to LDS, row by row: lane (n, g) has channels 2 W (4 g + i) + c of row n
    const float back = reach * (0x1p24f / kTop);
    if constexpr (SHARE) __syncthreads();                       // the area had the queries
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        l[j] += __shfl_xor(l[j], 16);
        l[j] += __shfl_xor(l[j], 32);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float *to = mine + n16 * kPad + 2 * W * (4 * g + i) + 2 * w;
                to[0] = (acc[j][2 * w][i] - ones[j][i]) * back;
                to[1] = (acc[j][2 * w + 1][i] * 0.0625f - ones[j][i]) * back;
            }
        if (g == 0) {
            row_max[wave][n16] = m[j];
            row_sum[wave][n16] = l[j];
        }
        if constexpr (SHARE) __syncthreads();
        else lanes_exchange_fence();
#pragma unroll
        for (int k = 0; k < (SHARE ? 1 : 4); ++k) {
            const int r = SHARE ? 4 * wave + g : 4 * k + g, row = row0 + 16 * j + r, first = n16 * C;
            float x[C], top, total;
            if constexpr (SHARE) {
                top = fmaxf(fmaxf(row_max[0][r], row_max[1][r]), fmaxf(row_max[2][r], row_max[3][r]));
                total = 0.0f;
#pragma unroll
                for (int i = 0; i < C; ++i) x[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float f = __builtin_amdgcn_exp2f(row_max[w][r] - top);
                    total = fmaf(f, row_sum[w][r], total);
#pragma unroll
                    for (int i = 0; i < C; ++i) x[i] = fmaf(f, area[w][r * kPad + first + i], x[i]);
                }
            } else {
                top = row_max[wave][r];
                total = row_sum[wave][r];
#pragma unroll
                for (int i = 0; i < C; ++i) x[i] = mine[r * kPad + first + i];
            }
            if (work.splits == 1) {
                if (row < rows) finish_row<D>(a, group, seq, head, row, x, total > 0.0f || total != total ? kv4_norm<D>() / total : 0.0f, lane);
            } else if (row < rows) {
                float *to = a.partials + partial_row(a, group, work.splits, b, head, row, split) * kPartial<D>;
#pragma unroll
                for (int i = 0; i < C / 2; ++i) reinterpret_cast<float2 *>(to + first)[i] = make_float2(x[2 * i], x[2 * i + 1]);
                if (n16 == 0) *reinterpret_cast<float2 *>(to + D) = make_float2(top, total);
            }
        }
        if constexpr (SHARE) __syncthreads();
        else lanes_exchange_fence();
    }
}

// The splits of a row put together: a block has a row, 16 lanes of it every sixteenth split.
template <int D>
__global__ __launch_bounds__(256) void kv4_join_kernel(Work work)
{
    constexpr int C = D / 16;
    __shared__ __align__(16) float sums[16][D + 4];
    __shared__ float tops[16], totals[16];
    const Kv4Attention &a = work.a;
    const int lane = threadIdx.x & 63, first = (lane & 15) * C, part = threadIdx.x >> 4, head = blockIdx.y, b = blockIdx.z, row = blockIdx.x;
    const Sequence seq = sequence_of(a, b);
    if (row >= seq.n * work.group) return;
    const int end = visible(a, seq, row / work.group), used = (end + work.chunk - 1) / work.chunk;
    const float *const from = a.partials + partial_row(a, work.group, work.splits, b, head, row, 0) * kPartial<D>;
    float top = kNone, total = 0.0f, x[C];
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = 0.0f;
    for (int s = part; s < used; s += 16) {
        const float *p = from + (size_t)s * kPartial<D>;
        const float2 end_of = *reinterpret_cast<const float2 *>(p + D);
        float y[C];
#pragma unroll
        for (int i = 0; i < C / 2; ++i) {
            const float2 v = reinterpret_cast<const float2 *>(p + first)[i];
            y[2 * i] = v.x;
            y[2 * i + 1] = v.y;
        }
        const float above = fmaxf(top, end_of.x), f = __builtin_amdgcn_exp2f(end_of.x - above), down = __builtin_amdgcn_exp2f(top - above);
        top = above;
        total = fmaf(f, end_of.y, total * down);
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] = fmaf(f, y[i], x[i] * down);
    }
#pragma unroll
    for (int i = 0; i < C; ++i) sums[part][first + i] = x[i];
    if ((lane & 15) == 0) {
        tops[part] = top;
        totals[part] = total;
    }
    __syncthreads();
    if (part != 0) return;
    top = tops[0];
#pragma unroll
    for (int p = 1; p < 16; ++p) top = fmaxf(top, tops[p]);
    total = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = 0.0f;
    for (int p = 0; p < min(used, 16); ++p) {
        const float f = __builtin_amdgcn_exp2f(tops[p] - top);
        total = fmaf(f, totals[p], total);
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] = fmaf(f, sums[p][first + i], x[i]);
    }
    finish_row<D>(a, work.group, seq, head, row, x, total > 0.0f || total != total ? kv4_norm<D>() / total : 0.0f, lane);
}

// How a call is cut up.
struct Plan {
    int tiles;          // of rows a block takes
    bool share;
    int nt, tiles_of_rows, chunk, splits;
};
Plan plan_of(int seqs, int max_q, int max_kv, int q_heads, int kv_heads)
{
    Plan p;
    const long long rows = (long long)max_q * (q_heads / kv_heads);
    p.share = rows <= 64;
    p.nt = p.share ? (rows <= 16 ? 1 : rows <= 32 ? 2 : 4) : 2;
    const int per_block = p.share ? 16 * p.nt : 64 * p.nt;
    p.tiles_of_rows = (int)((rows + per_block - 1) / per_block);
    const long long blocks = (long long)p.tiles_of_rows * kv_heads * seqs;
    // blocks that share rows: 512 fill the chip's registers once (131071 keys of one sequence: 32 us, 36 with 1024 blocks, 45 with 2048); the others are fewer than that only for few rows
    long long splits = (p.share ? 512 : 1024) / (blocks > 0 ? blocks : 1);
    const int least = p.share ? 128 : 512;
    const long long most = (max_kv + least - 1) / least;
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    p.chunk = (int)(((max_kv + splits - 1) / splits + least - 1) / least * least);
    if (p.chunk < least) p.chunk = least;
    p.splits = (max_kv + p.chunk - 1) / p.chunk;
    if (p.splits < 1) p.splits = 1;
    return p;
}

template <int D>
hipError_t launch(const Kv4Attention &a, hipStream_t stream)
{
    const Plan p = plan_of(a.seqs, a.max_q, a.max_kv, a.q_heads, a.pages.heads);
    const Work w{a, a.q_heads / a.pages.heads, p.chunk, p.splits};
    const dim3 grid(p.tiles_of_rows * p.splits, a.pages.heads, a.seqs);
    if (p.share && p.nt == 1) kv4_attention_kernel<D, 1, true><<<grid, 256, 0, stream>>>(w);
    else if (p.share && p.nt == 2) kv4_attention_kernel<D, 2, true><<<grid, 256, 0, stream>>>(w);
    else if (p.share) kv4_attention_kernel<D, 4, true><<<grid, 256, 0, stream>>>(w);
    else kv4_attention_kernel<D, 2, false><<<grid, 256, 0, stream>>>(w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    kv4_join_kernel<D><<<dim3(a.max_q * w.group, a.pages.heads, a.seqs), 256, 0, stream>>>(w);
    return hipGetLastError();
}

}  // namespace

size_t kv4_attention_workspace_bytes(int T, int seqs, int max_q, int max_kv, int q_heads, int kv_heads, int d)
{
    const Plan p = plan_of(seqs, max_q, max_kv, q_heads, kv_heads);
    return p.splits == 1 ? 0 : (size_t)seqs * q_heads * max_q * p.splits * (d + 2) * sizeof(float);
}

hipError_t run_kv4_attention(const Kv4Attention &a, int d, hipStream_t stream) { return d == 64 ? launch<64>(a, stream) : launch<128>(a, stream); }

}  // namespace qvggt

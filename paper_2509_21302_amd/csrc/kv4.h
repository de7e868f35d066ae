// A paged key/value cache held in 4 bits: where its bytes lie, and what the kernels that write and read it share.
//
// A page holds P tokens (a power of two from 16 to 1024) of every head; a head's part of a page is P * (D + 4) bytes, one after another:
//   the keys' codes     token after token, D / 2 bytes each: channel 2 j in the low half of byte j, 2 j + 1 in the high half
//   the values' codes   blocks of 16 tokens, 8 D bytes each: [4 groups of 4 tokens][16][D / 32][4 tokens] bytes; a byte is a pair of neighbouring channels of one
//                       token, pair p at [p / (D / 32)][p % (D / 32)]
//   the steps           4 bytes a token: the key's step as a bf16 in the low half, the value's in the high half
// Codes are kept as code + 8.  Both orders are those in which the lanes of a 16 x 16 x 32 matrix instruction want them, so that attention loads a block of 16 tokens as
// consecutive D / 8 bytes per lane and multiplies what it has loaded: in keys the lane of token t has a quarter of the channels, in values the lane of 16 channels
// (8 of them in D / 32 words) has a group of 4 tokens.  No byte has two tokens in it: a token is appended without reading its neighbours.
#pragma once
#include <type_traits>

#include "qvggt_common.h"

namespace qvggt {

constexpr int kKv4Block = 16;       // tokens of a block
inline bool kv4_valid_page(int page_tokens) { return page_tokens >= 16 && page_tokens <= 1024 && (page_tokens & (page_tokens - 1)) == 0; }
inline bool kv4_valid_head(int d) { return d == 64 || d == 128; }

struct Kv4Pages {
    uint8_t *base;
    int num_pages, page_shift, heads;      // P = 1 << page_shift
};
template <int D>
struct Kv4Layout {
    static constexpr int kRow = D / 2;              // bytes of a key
    static constexpr int kBlock = 8 * D;            // bytes of a block of 16 values
    static constexpr int kWords = D / 32;           // words of a lane's part of a block
    // byte offset of a head's part of a page
    __host__ __device__ static size_t part(int page, int head, int heads, int page_shift) { return ((size_t)page * heads + head) * ((size_t)(D + 4) << page_shift); }
    __host__ __device__ static int keys(int t) { return t * kRow; }
    __host__ __device__ static int values(int t, int page_shift) { return (kRow << page_shift) + (t >> 4) * kBlock; }
    __host__ __device__ static int steps(int t, int page_shift) { return (D << page_shift) + 4 * t; }
    // byte of channels 2 p and 2 p + 1 of token t (0 .. 15) inside a block of values
    __host__ __device__ static int value_byte(int t, int p) { return (((t >> 2) * 16 + p / kWords) * kWords + p % kWords) * 4 + (t & 3); }
};

// The rotation by position: pairs (c, c ^ pair) of the first `dim` channels, angle number (c / (2 pair)) * pair + c % pair of the row positions[token] of the
// table: [rows][cosines dim / 2, sines dim / 2].  table == nullptr: none.
struct Rope {
    const float *table;
    const int32_t *positions;
    int rows, dim, pair;
};

// ---- a row of D channels in 16 lanes, C = D / 16 consecutive channels in each, as it comes from memory: loads that depend on nothing first, those that need the
// position next, arithmetic last, so that a wave waits for memory twice and not once for every operand
template <int C>
struct HeadRow {
    // channels, and the ones they turn with where other lanes have those (bf16: half of the words).  All of it starts from something: what one path only sets would be kept in registers
    // from one turn of a surrounding loop to the next
    uint32_t x[C] = {}, partner[C] = {};
    float cosine[C] = {}, sine[C] = {};
    uint32_t sign[C / 4] = {};
    int at = 0;

    __device__ static void words(const void *row, bool f32, int first, uint32_t (&w)[C])
    {
        if (f32) {
#pragma unroll
            for (int i = 0; i < C / 4; ++i) {
                const uint4 v = reinterpret_cast<const uint4 *>(static_cast<const float *>(row) + first)[i];
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        } else if constexpr (C == 8) {
            const uint4 v = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(row) + first);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(row) + first);
            w[0] = v.x; w[1] = v.y;
        }
    }
    // The same of a row that nobody reads again: past the caches.
    __device__ static void words_once(const void *row, bool f32, int first, uint32_t (&w)[C])
    {
        typedef uint32_t Four __attribute__((ext_vector_type(4)));
        typedef uint32_t Half __attribute__((ext_vector_type(C / 2)));
        if (f32) {
#pragma unroll
            for (int i = 0; i < C / 4; ++i) {
                const Four v = __builtin_nontemporal_load(reinterpret_cast<const Four *>(static_cast<const float *>(row) + first) + i);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[4 * i + k] = v[k];
            }
        } else {
            const Half v = __builtin_nontemporal_load(reinterpret_cast<const Half *>(static_cast<const uint16_t *>(row) + first));
#pragma unroll
            for (int k = 0; k < C / 2; ++k) w[k] = v[k];
        }
    }
    __device__ static void floats(const uint32_t (&w)[C], bool f32, float (&y)[C])
    {
#pragma unroll
        for (int i = 0; i < C; ++i) y[i] = f32 ? __uint_as_float(w[i]) : __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    __device__ void load(const void *row, bool f32, int first, const int8_t *signs, bool once = false)
    {
        if (once) words_once(row, f32, first, x);
        else words(row, f32, first, x);
        if (signs != nullptr) {
#pragma unroll
            for (int i = 0; i < C / 4; ++i) sign[i] = reinterpret_cast<const uint32_t *>(signs + first)[i];
        }
    }
    __device__ void load_turn(const void *row, bool f32, int first, const Rope &rope, long long token)
    {
        if (rope.table == nullptr) return;
        at = rope.positions[token];
        if (rope.pair >= C) words(row, f32, first ^ rope.pair, partner);
    }
    __device__ void load_angles(int first, const Rope &rope)
    {
        if (rope.table == nullptr) return;
        // dim is a multiple of 16: a lane's channels turn or do not (those take the first ones' angles, for nothing).  C consecutive angles, or half as many where pairs are inside a lane
        const int c = first < rope.dim ? first : 0;
        const bool wide = rope.pair >= C;
        const int angle = wide ? (c / (2 * rope.pair)) * rope.pair + (c & (rope.pair - 1)) : c / 2;
        const float *from = rope.table + (size_t)min(max(at, 0), rope.rows - 1) * rope.dim + angle;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < C / 4; ++i) {
                const int k = (wide && h ? C / 2 : 0) + 2 * i, to = h * (C / 2) + 2 * i;
                const float2 u = *reinterpret_cast<const float2 *>(from + k), v = *reinterpret_cast<const float2 *>(from + rope.dim / 2 + k);
                cosine[to] = u.x; cosine[to + 1] = u.y;
                sine[to] = v.x; sine[to + 1] = v.y;
            }
    }
    __device__ void channels(bool f32, int first, const int8_t *signs, float (&y)[C]) const
    {
        floats(x, f32, y);
        if (signs != nullptr) flip(y);
    }
    // ... turned
    __device__ void turned(bool f32, int first, const Rope &rope, const int8_t *signs, float (&y)[C]) const
    {
        floats(x, f32, y);
        if (rope.table != nullptr) {
            const bool inside = first < rope.dim;
            float z[C];
            if (rope.pair >= C) {
                const float side = (first & rope.pair) ? 1.0f : -1.0f;
                float other[C];
                floats(partner, f32, other);
#pragma unroll
                for (int i = 0; i < C; ++i) z[i] = fmaf(y[i], cosine[i], side * sine[i] * other[i]);
            } else {
                auto within = [&](auto pair) {
                    constexpr int kPair = decltype(pair)::value;
#pragma unroll
                    for (int i = 0; i < C; ++i) {
                        constexpr int kAll = 2 * kPair;
                        const int angle = i / kAll * kPair + i % kPair;
                        z[i] = fmaf(y[i], cosine[angle], ((i & kPair) ? sine[angle] : -sine[angle]) * y[i ^ kPair]);
                    }
                };
                if (rope.pair == 1) within(std::integral_constant<int, 1>());
                else if (rope.pair == 2) within(std::integral_constant<int, 2>());
                else within(std::integral_constant<int, C / 2>());
            }
#pragma unroll
            for (int i = 0; i < C; ++i) y[i] = inside ? z[i] : y[i];
        }
        if (signs != nullptr) flip(y);
    }
    __device__ void flip(float (&y)[C]) const
    {
#pragma unroll
        for (int i = 0; i < C; ++i) y[i] = __uint_as_float(__float_as_uint(y[i]) ^ ((sign[i / 4] << (24 - 8 * (i % 4))) & 0x80000000u));
    }
};

template <int C>
__device__ inline void sign_channels(const int8_t *signs, int first, float (&x)[C])
{
    if (signs == nullptr) return;
#pragma unroll
    for (int i = 0; i < C / 4; ++i) {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(signs + first + 4 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * i + j] = __uint_as_float(__float_as_uint(x[4 * i + j]) ^ ((w << (24 - 8 * j)) & 0x80000000u));
    }
}

// The unnormalised Walsh-Hadamard butterflies of a row, the channel bits in rising order: those inside a lane, then the lane's four, as in lane_butterflies: the partner's value
// comes with the addition (DPP), the own one's sign is flipped before it
template <int CTRL>
__device__ inline float partner_of(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int C>
__device__ inline void row_butterflies(float (&x)[C], int lane)
{
#pragma unroll
    for (int b = 1; b < C; b *= 2)
#pragma unroll
        for (int i = 0; i < C; ++i)
            if (!(i & b)) {
                const float u = x[i], v = x[i | b];
                x[i] = u + v;
                x[i | b] = u - v;
            }
    const uint32_t s1 = (uint32_t)lane << 31, s2 = (uint32_t)(lane >> 1) << 31, s4 = (uint32_t)(lane >> 2) << 31, s8 = (uint32_t)(lane >> 3) << 31;
    auto flip = [](float v, uint32_t sign) { return __uint_as_float(__float_as_uint(v) ^ sign); };
#pragma unroll
    for (int r = 0; r < C; ++r) {
        x[r] = partner_of<0xB1>(x[r]) + flip(x[r], s1);
        x[r] = partner_of<0x4E>(x[r]) + flip(x[r], s2);
        x[r] = partner_of<0x141>(partner_of<0x1B>(x[r])) + flip(x[r], s4);
        x[r] = partner_of<0x128>(x[r]) + flip(x[r], s8);
    }
}

template <int D>
constexpr float kv4_norm() { return D == 64 ? 0.125f : 0.08838834764831845f; }       // 1 / sqrt(D)

// host side: the launchers behind the entry points
hipError_t run_kv4_append(const void *K, const void *V, bool f32, int T, long long k_stride, long long v_stride, int d, const Rope &rope, const int8_t *signs,
                          const int32_t *slots, const Kv4Pages &pages, hipStream_t stream);
hipError_t run_kv4_read(const Kv4Pages &pages, int d, const int32_t *slots, int T, const int8_t *signs, bool f32, void *K, void *V, hipStream_t stream);

struct Kv4Attention {
    const void *q;
    int q_f32, T, q_heads;
    long long q_stride;
    Rope rope;
    const int8_t *signs;
    float scale;
    int causal;
    Kv4Pages pages;
    const int32_t *table;
    int table_width;
    const int32_t *starts, *lens;
    int seqs, max_q, max_kv;
    uint16_t *out;
    void *workspace;
};
size_t kv4_attention_workspace_bytes(int seqs, int max_q, int max_kv, int q_heads, int kv_heads, int d);
hipError_t run_kv4_attention(const Kv4Attention &a, int d, hipStream_t stream);

}  // namespace qvggt

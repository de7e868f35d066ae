// The 4-bit key/value cache written and read back: qvggt_kv4_append and qvggt_kv4_read.
//
// A key is rotated by its position, a key or value x becomes z = (s * x) H / sqrt(D) (s random signs, H the Walsh-Hadamard matrix: one loud channel ends up spread over all
// of them), and z is rounded to 4-bit codes with one step per token and head.  16 lanes have a row of D channels: the butterflies are additions inside a lane and
// four DPP steps, the largest magnitude four more.
#include "kv4.h"

namespace qvggt {
namespace {

// codes + 8 of z, eight or four of them, channel i in bits 4 i .. 4 i + 3.  Turned rows of bf16 numbers have few bits, and quotients halfway between two codes are common (one
// in 10^5 of 64 channels): the product with the reciprocal is corrected by what it leaves over, which makes a quotient that is an fp32 number exact
template <int C>
__device__ inline uint32_t nibbles(const float (&z)[C], float step, float inv)
{
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        float t = z[i] * inv;
        t = fmaf(fmaf(-t, step, z[i]), inv, t);
        w |= (__float_as_uint(t + (kRoundMagic + 8.0f)) & 15u) << (4 * i);      // |t| <= 7 (1 + 2^-8): the code is in -7 .. 7
    }
    return w;
}

// z -> its step, rounded to bf16 (8 bits of a step that is uncertain by half a code: the codes are taken with the rounded step, so nothing else changes), and the codes.  A row with an
// infinity or no number in it, or whose sums overflow, has a step that is none: maxima here pass that on, and all that is read of the row shows it
template <int C>
__device__ inline uint32_t quantize(float (&z)[C], uint32_t *step_bits)
{
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) top = __builtin_elementwise_maximum(top, fabsf(z[i]));
    top = __builtin_elementwise_maximum(top, partner_of<0xB1>(top));            // over the row's 16 lanes, as max_over_16_lanes
    top = __builtin_elementwise_maximum(top, partner_of<0x4E>(top));
    top = __builtin_elementwise_maximum(top, partner_of<0x141>(top));
    top = __builtin_elementwise_maximum(top, partner_of<0x140>(top));
    const uint32_t bits = pack_bf16x2(top / 7.0f, 0.0f) & 0xffffu;
    const float step = bf16_bits_to_float(bits);
    const bool number = top < INFINITY, live = number && step >= kMinStep;
    *step_bits = live ? bits : number ? 0 : 0x7fc0u;
    return live ? nibbles<C>(z, step, 1.0f / step) : 0x88888888u >> (32 - 4 * C);
}

// Four tokens' bytes of values, a token in each of the lanes n, n + 16, n + 32, n + 48, become words of a pair of channels: lane n + 16 i then has byte i of all four.  Its own inverse.
// (64 channels: two bytes a token, words in lanes n and n + 16.)
__device__ inline uint32_t transpose_bytes(uint32_t w, int lane)
{
    auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);                      // the word of the lane below 32, and of the one above
    w = __builtin_amdgcn_perm(r[1], r[0], lane & 32 ? 0x07060302u : 0x05040100u);
    r = __builtin_amdgcn_permlane16_swap(w, w, false, false);                           // of the even row of 16 lanes, and of the odd one
    return __builtin_amdgcn_perm(r[1], r[0], lane & 16 ? 0x07030501u : 0x06020400u);
}

// What a wave has: tokens 4 unit - shift + (0 .. 3) of a head, 16 lanes each.  shift: what the first token's slot is past a group of four, so that a run of consecutive slots comes in
// whole groups; `whole`: this one is (its values are words of four tokens then, and bytes of one otherwise).
struct Quad {
    int head, slot, t, lane, first;
    long long token;
    bool there, whole;              // the lane's token is one of the call's; ...
    __device__ Quad(const int32_t *slots, int T, const Kv4Pages &pages, int C)
    {
        lane = threadIdx.x & 63;
        first = (lane & 15) * C;
        const unsigned unit = blockIdx.x * 4u + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), four = unit / (unsigned)pages.heads;
        head = (int)(unit - four * pages.heads);
        token = (long long)four * 4 - (slots[0] & 3) + (lane >> 4);
        there = token >= 0 && token < T;
        slot = there ? slots[token] : -1;
        there = there && slot >= 0 && slot < (long long)pages.num_pages << pages.page_shift;
        t = slot & ((1 << pages.page_shift) - 1);
        const int base = __builtin_amdgcn_readfirstlane(slot);
        whole = __builtin_amdgcn_ballot_w64(there && slot == base + (lane >> 4) && (base & 3) == 0) == ~0ull;
    }
};

// Keys and values of a quad's tokens.  16411 tokens of 8 heads x 128 channels in f32, 152 MB: 40 us, 3.8 TB/s; bound by ~600 vector instructions a wave (0.74 of the cycles issue one) and by the chain
// slots, positions, angles and rows.  Few tokens: that chain alone (one token 3.5 us with its launch).  The values' rows are read past the caches (47 us for 44 within them); the keys' are not:
// a channel and its partner read the same row.
template <int D, bool f32>
__global__ __launch_bounds__(256) void kv4_append_kernel(const void *K, const void *V, int T, long long k_stride, long long v_stride, Rope rope, const int8_t *signs,
                                                         const int32_t *slots, Kv4Pages pages)
{
    using L = Kv4Layout<D>;
    constexpr int C = D / 16;
    const Quad q(slots, T, pages, C);
    constexpr int elem = f32 ? 4 : 2;
    const long long token = min(max(q.token, 0LL), (long long)T - 1);                   // (lanes without a token load one, and store nothing)
    const char *k_row = static_cast<const char *>(K) + (token * k_stride + (long long)q.head * D) * elem, *v_row = static_cast<const char *>(V) + (token * v_stride + (long long)q.head * D) * elem;
    HeadRow<C> key, value;
    key.load(k_row, f32, q.first, signs);
    key.load_turn(k_row, f32, q.first, rope, token);
    value.load(v_row, f32, q.first, signs, true);
    key.load_angles(q.first, rope);
    uint32_t w[2], step[2];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float x[C];
        if (which == 0) value.channels(f32, q.first, signs, x);                         // values first: the keys' angles are on their way
        else key.turned(f32, q.first, rope, signs, x);
        row_butterflies<C>(x, q.lane);
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] *= kv4_norm<D>();
        w[which] = quantize<C>(x, &step[which]);
    }
    const uint32_t bytes = transpose_bytes(w[0], q.lane);
    if (!q.there) return;
    uint8_t *const part = pages.base + L::part(q.slot >> pages.page_shift, q.head, pages.heads, pages.page_shift);
    uint8_t *const k_to = part + L::keys(q.t) + q.first / 2, *const v_to = part + L::values(q.t, pages.page_shift);
    if constexpr (C == 8) *reinterpret_cast<uint32_t *>(k_to) = w[1];
    else *reinterpret_cast<uint16_t *>(k_to) = (uint16_t)w[1];
    if (q.whole) {
        const int i = q.lane >> 4;
        if (C == 8 || i < 2) *reinterpret_cast<uint32_t *>(v_to + L::value_byte(q.t & 12, q.first / 2 + i)) = bytes;
    } else {
#pragma unroll
        for (int i = 0; i < C / 2; ++i) v_to[L::value_byte(q.t & 15, q.first / 2 + i)] = (uint8_t)(w[0] >> (8 * i));
    }
    if ((q.lane & 15) == 0) *reinterpret_cast<uint32_t *>(part + L::steps(q.t, pages.page_shift)) = step[1] | step[0] << 16;
}

template <int C>
__device__ inline void store_channels(void *row, bool f32, int first, const float (&x)[C])
{
    if (f32) {
#pragma unroll
        for (int i = 0; i < C / 4; ++i) {
            typedef float Four __attribute__((ext_vector_type(4)));
            __builtin_nontemporal_store(Four{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]}, reinterpret_cast<Four *>(static_cast<float *>(row) + first) + i);
        }
    } else {
        typedef uint32_t Half __attribute__((ext_vector_type(C / 2)));
        Half v;
#pragma unroll
        for (int i = 0; i < C / 2; ++i) v[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
        __builtin_nontemporal_store(v, reinterpret_cast<Half *>(static_cast<uint16_t *>(row) + first));
    }
}

// What a quad's tokens hold: codes times step, turned back.  The same 16411 tokens into bf16, 84 MB: 22 us, 3.8 TB/s, with a vector instruction issuing in 0.78 of the cycles; the rows leave past the
// caches (24 us for 23 through them).
template <int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Pages pages, const int32_t *slots, int T, const int8_t *signs, bool f32, void *K, void *V)
{
    using L = Kv4Layout<D>;
    constexpr int C = D / 16;
    const Quad q(slots, T, pages, C);
    const uint8_t *const part = pages.base + (q.there ? L::part(q.slot >> pages.page_shift, q.head, pages.heads, pages.page_shift) : 0);
    uint32_t w[2] = {}, steps = 0;
    if (q.there) {
        steps = *reinterpret_cast<const uint32_t *>(part + L::steps(q.t, pages.page_shift));
        const uint8_t *const k_from = part + L::keys(q.t) + q.first / 2, *const v_from = part + L::values(q.t, pages.page_shift);
        if constexpr (C == 8) w[0] = *reinterpret_cast<const uint32_t *>(k_from);
        else w[0] = *reinterpret_cast<const uint16_t *>(k_from);
        if (q.whole) {
            const int i = C == 8 ? q.lane >> 4 : q.lane >> 4 & 1;                       // (64 channels: lanes from 32 on load a word for nothing)
            w[1] = *reinterpret_cast<const uint32_t *>(v_from + L::value_byte(q.t & 12, q.first / 2 + i));
        } else {
#pragma unroll
            for (int i = 0; i < C / 2; ++i) w[1] |= (uint32_t)v_from[L::value_byte(q.t & 15, q.first / 2 + i)] << (8 * i);
        }
    }
    if (q.whole) w[1] = transpose_bytes(w[1], q.lane);
    if (q.token < 0 || q.token >= T) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        void *out = which ? V : K;
        if (out == nullptr) continue;
        const float step = (which ? __uint_as_float(steps & 0xffff0000u) : bf16_bits_to_float(steps & 0xffffu)) * kv4_norm<D>();
        float x[C];
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] = q.there ? (float)((int)(w[which] >> (4 * i) & 15u) - 8) * step : 0.0f;
        row_butterflies<C>(x, q.lane);
        sign_channels<C>(signs, q.first, x);
        char *row = static_cast<char *>(out) + ((q.token * pages.heads + q.head) * D) * (f32 ? 4 : 2);
        store_channels<C>(row, f32, q.first, x);
    }
}

// blocks of four quads: one quad more than the tokens fill, for the shift
unsigned quad_blocks(int T, int heads) { return (unsigned)((((long long)T + 3 + 3) / 4 * heads + 3) / 4); }

}  // namespace

hipError_t run_kv4_append(const void *K, const void *V, bool f32, int T, long long k_stride, long long v_stride, int d, const Rope &rope, const int8_t *signs,
                          const int32_t *slots, const Kv4Pages &pages, hipStream_t stream)
{
    const dim3 grid(quad_blocks(T, pages.heads));
    auto launch = [&](auto kernel) { kernel<<<grid, 256, 0, stream>>>(K, V, T, k_stride, v_stride, rope, signs, slots, pages); };
    if (d == 64) launch(f32 ? kv4_append_kernel<64, true> : kv4_append_kernel<64, false>);
    else launch(f32 ? kv4_append_kernel<128, true> : kv4_append_kernel<128, false>);
    return hipGetLastError();
}

hipError_t run_kv4_read(const Kv4Pages &pages, int d, const int32_t *slots, int T, const int8_t *signs, bool f32, void *K, void *V, hipStream_t stream)
{
    const dim3 grid(quad_blocks(T, pages.heads));
    if (d == 64) kv4_read_kernel<64><<<grid, 256, 0, stream>>>(pages, slots, T, signs, f32, K, V);
    else kv4_read_kernel<128><<<grid, 256, 0, stream>>>(pages, slots, T, signs, f32, K, V);
    return hipGetLastError();
}

}  // namespace qvggt

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

// z -> its step, rounded to bf16 (8 bits of a step that is uncertain by half a code: the codes are taken with the rounded step, so nothing else changes), and the codes
template <int C>
__device__ inline uint32_t quantize(float (&z)[C], uint32_t *step_bits)
{
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) top = fmaxf(top, fabsf(z[i]));
    top = max_over_16_lanes(top);
    const uint32_t bits = pack_bf16x2(top / 7.0f, 0.0f) & 0xffffu;
    const float step = bf16_bits_to_float(bits);
    const bool live = step >= kMinStep;
    *step_bits = live ? bits : 0;
    return nibbles<C>(z, step, live ? 1.0f / step : 0.0f);
}

// A wave has four tokens of one head, 16 lanes each; keys first, then values.
template <int D>
__global__ __launch_bounds__(256) void kv4_append_kernel(const void *K, const void *V, bool f32, int T, long long k_stride, long long v_stride, Rope rope, const int8_t *signs,
                                                         const int32_t *slots, Kv4Pages pages)
{
    using L = Kv4Layout<D>;
    constexpr int C = D / 16;
    const int lane = threadIdx.x & 63, first = (lane & 15) * C;
    const long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int head = (int)(unit % pages.heads);
    const long long token = unit / pages.heads * 4 + (lane >> 4);
    if (token >= T) return;
    const int slot = slots[token];
    if (slot < 0 || slot >= (long long)pages.num_pages << pages.page_shift) return;
    const int elem = f32 ? 4 : 2, t = slot & ((1 << pages.page_shift) - 1);
    uint8_t *const part = pages.base + L::part(slot >> pages.page_shift, head, pages.heads, pages.page_shift);
    const char *k_row = static_cast<const char *>(K) + (token * k_stride + (long long)head * D) * elem, *v_row = static_cast<const char *>(V) + (token * v_stride + (long long)head * D) * elem;
    HeadRow<C> key, value;
    key.load(k_row, f32, first, signs);
    key.load_turn(k_row, f32, first, rope, token);
    value.load(v_row, f32, first, signs);
    key.load_angles(first, rope);
    uint32_t steps = 0;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float x[C];
        if (which == 0) key.turned(f32, first, rope, signs, x);
        else value.channels(f32, first, signs, x);
        row_butterflies<C>(x, lane);
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] *= kv4_norm<D>();
        uint32_t step;
        const uint32_t w = quantize<C>(x, &step);
        steps |= step << (16 * which);
        if (which == 0) {
            uint8_t *to = part + L::keys(t) + first / 2;
            if constexpr (C == 8) *reinterpret_cast<uint32_t *>(to) = w;
            else *reinterpret_cast<uint16_t *>(to) = (uint16_t)w;
        } else {
            uint8_t *to = part + L::values(t, pages.page_shift);
#pragma unroll
            for (int i = 0; i < C / 2; ++i) to[L::value_byte(t & 15, first / 2 + i)] = (uint8_t)(w >> (8 * i));
        }
    }
    if ((lane & 15) == 0) *reinterpret_cast<uint32_t *>(part + L::steps(t, pages.page_shift)) = steps;
}

template <int C>
__device__ inline void store_channels(void *row, bool f32, int first, const float (&x)[C])
{
    if (f32) {
#pragma unroll
        for (int i = 0; i < C / 4; ++i) reinterpret_cast<float4 *>(static_cast<float *>(row) + first)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < C / 4; ++i) reinterpret_cast<uint2 *>(static_cast<uint16_t *>(row) + first)[i] = make_uint2(pack_bf16x2(x[4 * i], x[4 * i + 1]), pack_bf16x2(x[4 * i + 2], x[4 * i + 3]));
    }
}

// 16 lanes have a token of a head: codes times step, turned back
template <int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Pages pages, const int32_t *slots, int T, const int8_t *signs, bool f32, void *K, void *V)
{
    using L = Kv4Layout<D>;
    constexpr int C = D / 16;
    const int lane = threadIdx.x & 63, first = (lane & 15) * C;
    const long long unit = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
    const long long token = unit / pages.heads;
    if (token >= T) return;
    const int head = (int)(unit % pages.heads), slot = slots[token], t = slot & ((1 << pages.page_shift) - 1);
    const bool held = slot >= 0 && slot < (long long)pages.num_pages << pages.page_shift;
    const uint8_t *const part = pages.base + (held ? L::part(slot >> pages.page_shift, head, pages.heads, pages.page_shift) : 0);
    const uint32_t steps = held ? *reinterpret_cast<const uint32_t *>(part + L::steps(t, pages.page_shift)) : 0;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        void *out = which ? V : K;
        if (out == nullptr) continue;
        uint32_t w = 0;
        if (held) {
            if (which == 0) {
                const uint8_t *from = part + L::keys(t) + first / 2;
                if constexpr (C == 8) w = *reinterpret_cast<const uint32_t *>(from);
                else w = *reinterpret_cast<const uint16_t *>(from);
            } else {
                const uint8_t *from = part + L::values(t, pages.page_shift);
#pragma unroll
                for (int i = 0; i < C / 2; ++i) w |= (uint32_t)from[L::value_byte(t & 15, first / 2 + i)] << (8 * i);
            }
        }
        const float step = (which ? __uint_as_float(steps & 0xffff0000u) : bf16_bits_to_float(steps & 0xffffu)) * kv4_norm<D>();
        float x[C];
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] = held ? (float)((int)(w >> (4 * i) & 15u) - 8) * step : 0.0f;
        row_butterflies<C>(x, lane);
        sign_channels<C>(signs, first, x);
        char *row = static_cast<char *>(out) + ((token * pages.heads + head) * D) * (f32 ? 4 : 2);
        store_channels<C>(row, f32, first, x);
    }
}

}  // namespace

hipError_t run_kv4_append(const void *K, const void *V, bool f32, int T, long long k_stride, long long v_stride, int d, const Rope &rope, const int8_t *signs,
                          const int32_t *slots, const Kv4Pages &pages, hipStream_t stream)
{
    const long long units = ((long long)T + 3) / 4 * pages.heads;
    const dim3 grid((unsigned)((units + 3) / 4));
    if (d == 64) kv4_append_kernel<64><<<grid, 256, 0, stream>>>(K, V, f32, T, k_stride, v_stride, rope, signs, slots, pages);
    else kv4_append_kernel<128><<<grid, 256, 0, stream>>>(K, V, f32, T, k_stride, v_stride, rope, signs, slots, pages);
    return hipGetLastError();
}

hipError_t run_kv4_read(const Kv4Pages &pages, int d, const int32_t *slots, int T, const int8_t *signs, bool f32, void *K, void *V, hipStream_t stream)
{
    const dim3 grid((unsigned)(((long long)T * pages.heads + 15) / 16));
    if (d == 64) kv4_read_kernel<64><<<grid, 256, 0, stream>>>(pages, slots, T, signs, f32, K, V);
    else kv4_read_kernel<128><<<grid, 256, 0, stream>>>(pages, slots, T, signs, f32, K, V);
    return hipGetLastError();
}

}  // namespace qvggt

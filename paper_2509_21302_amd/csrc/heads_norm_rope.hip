// Heads of queries and keys, as they lie in the rows of a fused product: norm over a head's channels, gain and bias, rotation by positions with several axes.
//
// d / 8 lanes have a head, eight channels each, and a wave has heads of one token: what turns them (the token's positions, its rows of the table) is loaded once for all of its heads.  Means and
// variances are two passes over registers, sums between lanes by DPP, and so are the channels that a lane's own turn with.
#include "block_rows.h"

namespace qvggt {
namespace {

constexpr int kAtOnce = 4;      // heads of a lane whose loads are in flight together

template <int LANES>
__device__ inline float sum_over(float v)
{
    v = dpp_add_step<0xB1>(v);
    v = dpp_add_step<0x4E>(v);
    v = dpp_add_step<0x141>(v);
    return LANES == 8 ? v : dpp_add_step<0x140>(v);
}

template <int D>
__global__ __launch_bounds__(256) void heads_norm_rope_kernel(HeadsNormRope a, int span, int chunks_q, int chunks)
{
    constexpr int kLanes = D / 8, kGroups = 64 / kLanes;
    const int lane = threadIdx.x & 63, id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token = id / chunks, chunk = id % chunks;
    if (token >= a.T) return;
    const int which = chunk >= chunks_q, first = (lane % kLanes) * 8;
    const int heads = which ? a.heads[1] : a.heads[0], from = (which ? chunk - chunks_q : chunk) * span * kGroups, head0 = from + lane / kLanes, stop = min(from + span * kGroups, heads);
    const bool f32 = a.f32;
    const size_t size = f32 ? 4 : 2;
    const char *const in = static_cast<const char *>(which ? a.in[1] : a.in[0]) + size * token * (which ? a.in_stride[1] : a.in_stride[0]);
    char *const out = static_cast<char *>(which ? a.out[1] : a.out[0]) + size * token * (which ? a.out_stride[1] : a.out_stride[0]);

    // The angles of this lane's channels: eight cosines and sines, or four where channels turn with others of the lane
    const bool turns = a.rope != nullptr && first < a.dim, wide = a.pair >= 8;
    float cosine[8], sine[8];
    if (a.rope != nullptr) {
        const int c = turns ? first : 0, half = a.dim / 2;
        const int p0 = wide ? c / (2 * a.pair) * a.pair + (c & (a.pair - 1)) : c / 2;
        int at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = i < a.axes ? min(max(a.positions[(size_t)i * a.T + token], 0), a.rows - 1) : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i >= 4 && !wide) break;
            const int p = p0 + i, section = p * a.axes;
            const int axis = min(a.pair_axis != nullptr ? a.pair_axis[p] : (section >= half) + (section >= 2 * half) + (section >= 3 * half), a.axes - 1);
            const int row = axis == 0 ? at[0] : axis == 1 ? at[1] : axis == 2 ? at[2] : at[3];
            const float *const angle = a.rope + (size_t)row * a.dim + p;
            cosine[i] = angle[0];
            sine[i] = angle[half];
        }
    }
    float gain[8], bias[8];
    const float *const g = which ? a.gain[1] : a.gain[0], *const b = which ? a.bias[1] : a.bias[0];
    if (g != nullptr) load_eight(g + first, gain);
    if (b != nullptr) load_eight(b + first, bias);

    for (int h0 = head0; h0 < stop; h0 += kAtOnce * kGroups) {
        Eight raw[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) raw[k].load(in + size * D * min(h0 + k * kGroups, stop - 1), f32, first);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            float y[8];
            raw[k].floats(f32, y);
            if (a.norm != kNormNone) {
                if (a.norm == kNormLayer) {
                    float s = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) s += y[i];
                    const float mean = sum_over<kLanes>(s) * (1.0f / D);
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] -= mean;
                }
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) s = fmaf(y[i], y[i], s);
                const float f = inverse_root(sum_over<kLanes>(s) * (1.0f / D) + a.eps);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] *= f;
            }
            if (g != nullptr)
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] *= gain[i];
            if (b != nullptr)
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] += bias[i];
            if (a.rope != nullptr) {
                float z[8];
                auto across = [&](auto other) {
                    const float side = first & a.pair ? 1.0f : -1.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[i] = fmaf(y[i], cosine[i], side * sine[i] * other(y[i]));
                };
                auto within = [&](auto pair) {
                    constexpr int kPair = decltype(pair)::value;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        constexpr int kAll = 2 * kPair;
                        const int angle = i / kAll * kPair + i % kPair;
                        z[i] = fmaf(y[i], cosine[angle], (i & kPair ? sine[angle] : -sine[angle]) * y[i ^ kPair]);
                    }
                };
                switch (a.pair) {
                    case 1: within(std::integral_constant<int, 1>()); break;
                    case 2: within(std::integral_constant<int, 2>()); break;
                    case 4: within(std::integral_constant<int, 4>()); break;
                    case 8: across([](float v) { return dpp_move<0xB1>(v); }); break;
                    case 16: across([](float v) { return dpp_move<0x4E>(v); }); break;
                    case 32: across([](float v) { return dpp_move<0x141>(dpp_move<0x1B>(v)); }); break;
                    default: across([](float v) { return dpp_move<0x128>(v); }); break;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = turns ? z[i] : y[i];
            }
            if (h0 + k * kGroups < stop) store_eight(out + size * D * (h0 + k * kGroups), f32, first, y);
        }
    }
}

template <int D>
hipError_t launch(const HeadsNormRope &a, hipStream_t stream)
{
    constexpr int kGroups = 64 / (D / 8);
    const int span = kAtOnce;
    const int chunks_q = (a.heads[0] + span * kGroups - 1) / (span * kGroups), chunks = chunks_q + (a.heads[1] + span * kGroups - 1) / (span * kGroups);
    heads_norm_rope_kernel<D><<<dim3((unsigned)(((long long)a.T * chunks + 3) / 4)), 256, 0, stream>>>(a, span, chunks_q, chunks);
    return hipGetLastError();
}

}  // namespace

hipError_t run_heads_norm_rope(const HeadsNormRope &a, int d, hipStream_t stream) { return d == 64 ? launch<64>(a, stream) : launch<128>(a, stream); }

}  // namespace qvggt

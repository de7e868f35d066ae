// Heads of queries and keys, as they lie in the rows of a fused product: norm over a head's channels, gain and bias, rotation by positions with several axes.
//
// d / 8 lanes have a head, eight channels each, and a wave has heads of one token: what turns them (the token's positions, its rows of the table) is loaded once for all of its heads.  Means and
// variances are two passes over registers, sums between lanes by DPP, and so are the channels that a lane's own turn with.
#include "block_rows.h"

namespace qvggt {
namespace {

template <int LANES>
__device__ inline float sum_over(float v)
{
    v = dpp_add_step<0xB1>(v);
    v = dpp_add_step<0x4E>(v);
    v = dpp_add_step<0x141>(v);
    return LANES == 8 ? v : dpp_add_step<0x140>(v);
}

// HEADS: of a lane, whose loads are in flight together.  Chunks of a token: of queries first, of keys then.
template <int D, bool F32, int HEADS>
__global__ __launch_bounds__(256) void heads_norm_rope_kernel(HeadsNormRope a, int chunks_q, int chunks)
{
    constexpr int kLanes = D / 8, kGroups = 64 / kLanes, kSize = F32 ? 4 : 2;
    const int lane = threadIdx.x & 63, id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token = id / chunks, chunk = id % chunks;
    if (token >= a.T) return;
    const bool of_keys = chunk >= chunks_q;
    const int first = (lane % kLanes) * 8, heads = of_keys ? a.heads[1] : a.heads[0], head0 = (of_keys ? chunk - chunks_q : chunk) * HEADS * kGroups + lane / kLanes;
    const char *const in = static_cast<const char *>(of_keys ? a.in[1] : a.in[0]) + kSize * token * (of_keys ? a.in_stride[1] : a.in_stride[0]);
    char *const out = static_cast<char *>(of_keys ? a.out[1] : a.out[0]) + kSize * token * (of_keys ? a.out_stride[1] : a.out_stride[0]);
    const float *const g = of_keys ? a.gain[1] : a.gain[0], *const b = of_keys ? a.bias[1] : a.bias[0];
    Eight<F32> raw[HEADS];
#pragma unroll
    for (int k = 0; k < HEADS; ++k) raw[k].load(in + (size_t)kSize * D * min(head0 + k * kGroups, heads - 1), first);
    float gain[8], bias[8];
    if (g != nullptr) load_eight(g + first, gain);
    if (b != nullptr) load_eight(b + first, bias);

    // The angles of this lane's channels: eight cosines and sines, or four where channels turn with others of the lane
    const bool turns = a.rope != nullptr && first < a.dim, wide = a.pair >= 8;
    float cosine[8], sine[8];
    if (a.rope != nullptr) {
        const int c = turns ? first : 0, half = a.dim / 2;
        const int p0 = wide ? c / (2 * a.pair) * a.pair + (c & (a.pair - 1)) : c / 2;
        int at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = i < a.axes ? min(max(a.positions[(size_t)i * a.T + token], 0), a.rows - 1) : 0;
        auto axis_of = [&](int p) {
            const int section = p * a.axes;
            return min(a.pair_axis != nullptr ? a.pair_axis[p] : (section >= half) + (section >= 2 * half) + (section >= 3 * half), a.axes - 1);
        };
        auto row_of = [&](int axis) { return axis == 0 ? at[0] : axis == 1 ? at[1] : axis == 2 ? at[2] : at[3]; };
        if (wide && (a.axes == 1 || (a.pair_axis == nullptr && half % (8 * a.axes) == 0))) {        // the angles of one row
            const float *const angle = a.rope + (size_t)row_of(a.axes == 1 ? 0 : axis_of(p0)) * a.dim + p0;
            load_eight(angle, cosine);
            load_eight(angle + half, sine);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i >= 4 && !wide) break;
                const float *const angle = a.rope + (size_t)row_of(axis_of(p0 + i)) * a.dim + p0 + i;
                cosine[i] = angle[0];
                sine[i] = angle[half];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < HEADS; ++k) {
        float y[8];
        raw[k].floats(y);
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
        if (head0 + k * kGroups < heads) store_eight<F32>(out + (size_t)kSize * D * (head0 + k * kGroups), first, y);
    }
}

template <int D, bool F32, int HEADS>
hipError_t launch(const HeadsNormRope &a, hipStream_t stream)
{
    constexpr int kGroups = 64 / (D / 8);
    const int chunks_q = (a.heads[0] + HEADS * kGroups - 1) / (HEADS * kGroups), chunks = chunks_q + (a.heads[1] + HEADS * kGroups - 1) / (HEADS * kGroups);
    heads_norm_rope_kernel<D, F32, HEADS><<<dim3((unsigned)(((long long)a.T * chunks + 3) / 4)), 256, 0, stream>>>(a, chunks_q, chunks);
    return hipGetLastError();
}
// Four heads a lane, or fewer where there are no more
template <int D, bool F32>
hipError_t launch(const HeadsNormRope &a, hipStream_t stream)
{
    const int most = (a.heads[0] > a.heads[1] ? a.heads[0] : a.heads[1]) * (D / 8);
    if (most <= 64) return launch<D, F32, 1>(a, stream);
    if (most <= 128) return launch<D, F32, 2>(a, stream);
    return launch<D, F32, 4>(a, stream);
}

}  // namespace

hipError_t run_heads_norm_rope(const HeadsNormRope &a, int d, hipStream_t stream)
{
    if (d == 64) return a.f32 ? launch<64, true>(a, stream) : launch<64, false>(a, stream);
    return a.f32 ? launch<128, true>(a, stream) : launch<128, false>(a, stream);
}

}  // namespace qvggt

// Heads of queries and keys, as they lie in the rows of a fused product: norm over a head's channels, gain and bias, rotation by positions with several axes.
//
// d / 8 lanes have a head, eight channels each, and a wave has heads of one token: what turns them (the token's positions, its rows of the table) is found once for all of them, one pair of channels
// a lane, and handed out through LDS (16411 tokens of 32 + 8 heads x 128 in float32, three axes whose pairs take turns: 134 us; 164 with every lane finding all of its own).  Means and variances are two
// passes over registers, sums between lanes by DPP, and so are the channels that a lane's own turn with.  Bound by memory: 5.1 TB/s there, 5.6 on ten frames (13740 tokens of 16 + 16 heads x 64 in
// bf16: 20 us), read and written, where a copy reaches 4.7 to 5.4 by its size.
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

// HEADS: of a lane, whose loads are in flight together: a chunk.  A token's chunks are those of its queries, then those of its keys; a wave has `each` of them.
template <int D, bool F32, int HEADS>
__global__ __launch_bounds__(256) void heads_norm_rope_kernel(HeadsNormRope a, int chunks_q, int chunks, int each)
{
    constexpr int kLanes = D / 8, kGroups = 64 / kLanes, kSize = F32 ? 4 : 2;
    __shared__ __align__(16) float angles[4][2][D / 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = (chunks + each - 1) / each;
    const int id = blockIdx.x * 4 + wave, token = id / waves, chunk0 = id % waves * each, stop = min(chunk0 + each, chunks);
    if (token >= a.T) return;
    const int first = (lane % kLanes) * 8, group = lane / kLanes;
    struct Place {
        bool of_keys;
        int head0, heads;
    };
    auto place = [&](int chunk) {
        const bool of_keys = chunk >= chunks_q;
        return Place{of_keys, (of_keys ? chunk - chunks_q : chunk) * HEADS * kGroups + group, of_keys ? a.heads[1] : a.heads[0]};
    };
    Eight<F32> next[HEADS];
    auto load = [&](int chunk) {
        const Place p = place(chunk);
        const char *const in = static_cast<const char *>(p.of_keys ? a.in[1] : a.in[0]) + kSize * token * (p.of_keys ? a.in_stride[1] : a.in_stride[0]);
#pragma unroll
        for (int k = 0; k < HEADS; ++k) next[k].load(in + (size_t)kSize * D * min(p.head0 + k * kGroups, p.heads - 1), first);
    };
    load(chunk0);

    // A lane finds the angle of one pair of channels; through LDS, where every lane then has those of its channels: eight cosines and sines, or four where channels turn with others of the lane
    const bool turns = a.rope != nullptr && first < a.dim, wide = a.pair >= 8;
    float cosine[8], sine[8];
    if (a.rope != nullptr) {
        const int half = a.dim / 2;
        if (lane < half) {
            const int section = lane * a.axes;
            const int axis = min(a.pair_axis != nullptr ? a.pair_axis[lane] : (section >= half) + (section >= 2 * half) + (section >= 3 * half), a.axes - 1);
            const float *const angle = a.rope + (size_t)min(max(a.positions[(size_t)axis * a.T + token], 0), a.rows - 1) * a.dim + lane;
            angles[wave][0][lane] = angle[0];
            angles[wave][1][lane] = angle[half];
        }
        lanes_exchange_fence();
        const int c = turns ? first : 0;
        const int p0 = wide ? c / (2 * a.pair) * a.pair + (c & (a.pair - 1)) : c / 2;
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const int p = p0 + (wide ? i : 0);              // (the second four are nobody's where pairs are inside a lane)
            const float4 u = *reinterpret_cast<const float4 *>(&angles[wave][0][p]), v = *reinterpret_cast<const float4 *>(&angles[wave][1][p]);
            cosine[i] = u.x; cosine[i + 1] = u.y; cosine[i + 2] = u.z; cosine[i + 3] = u.w;
            sine[i] = v.x; sine[i + 1] = v.y; sine[i + 2] = v.z; sine[i + 3] = v.w;
        }
    }
    float gain[8], bias[8];
    const float *g = nullptr, *b = nullptr;
    for (int chunk = chunk0; chunk < stop; ++chunk) {
        const Place here = place(chunk);
        char *const out = static_cast<char *>(here.of_keys ? a.out[1] : a.out[0]) + kSize * token * (here.of_keys ? a.out_stride[1] : a.out_stride[0]);
        if (chunk == chunk0 || chunk == chunks_q) {
            g = here.of_keys ? a.gain[1] : a.gain[0];
            b = here.of_keys ? a.bias[1] : a.bias[0];
            if (g != nullptr) load_eight(g + first, gain);
            if (b != nullptr) load_eight(b + first, bias);
        }
        Eight<F32> raw[HEADS];
#pragma unroll
        for (int k = 0; k < HEADS; ++k) raw[k] = next[k];
        if (chunk + 1 < stop) load(chunk + 1);
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
            if (here.head0 + k * kGroups < here.heads) store_eight<F32>(out + (size_t)kSize * D * (here.head0 + k * kGroups), first, y);
        }
    }
}

template <int D, bool F32, int HEADS>
hipError_t launch(const HeadsNormRope &a, hipStream_t stream)
{
    constexpr int kGroups = 64 / (D / 8);
    const int chunks_q = (a.heads[0] + HEADS * kGroups - 1) / (HEADS * kGroups), chunks = chunks_q + (a.heads[1] + HEADS * kGroups - 1) / (HEADS * kGroups);
    // All of a token's chunks where there are tokens enough for all waves of the chip: 13740 tokens of 16 + 16 heads x 64 in bf16 21.5 us for 24.8 with a wave for every chunk; 4096 of 32 + 8 x 128 in float32 34.4
    // for 37.8, 2048 21.2 both, 1024 13.2 for 11.8.  (In bf16 these meet at 6000 tokens: 8192 37.5 for 38.5, 2048 13.2 for 12.3, 1024 10.0 for 7.8.)
    const int each = a.T >= 2048 ? chunks : 1, waves = (chunks + each - 1) / each;
    heads_norm_rope_kernel<D, F32, HEADS><<<dim3((unsigned)(((long long)a.T * waves + 3) / 4)), 256, 0, stream>>>(a, chunks_q, chunks, each);
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

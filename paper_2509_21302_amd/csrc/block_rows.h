// The row operators around a block's layers: heads of queries and keys normalised and rotated, and the residual stream's update with its norms.
#pragma once
#include <type_traits>

#include "qvggt_common.h"

namespace qvggt {

enum { kNormNone = 0, kNormLayer = 1, kNormRms = 2 };

struct HeadsNormRope {
    const void *in[2];              // queries, keys
    void *out[2];
    long long in_stride[2], out_stride[2];
    int heads[2];
    const float *gain[2], *bias[2];
    int T, f32, norm;
    float eps;
    const float *rope;              // [rows][cosines dim / 2, sines dim / 2], or nullptr
    int rows, dim, pair, axes;
    const int32_t *positions;       // [axes][T]
    const uint8_t *pair_axis;       // [dim / 2], or nullptr: axis p * axes / (dim / 2)
};
hipError_t run_heads_norm_rope(const HeadsNormRope &a, int d, hipStream_t stream);

struct ResidualNorm {
    const void *x, *y;
    int x_f32, y_f32, M, C, post_norm;
    const float *post_gain, *post_bias, *scale;
    const void *gate;
    int norm;
    const float *gain, *bias;
    const void *mod_scale, *mod_shift;
    int cond_f32, cond_rows;
    long long cond_stride;
    const int32_t *row_of;
    float eps;
    void *x_out, *h;
    int h_f32;
};
hipError_t run_residual_norm(const ResidualNorm &a, hipStream_t stream);

// ---- eight consecutive channels of a row, as they come from memory
template <bool F32>
struct Eight {
    uint4 w[F32 ? 2 : 1];

    __device__ void load(const void *row, int first)
    {
        const uint4 *const from = reinterpret_cast<const uint4 *>(static_cast<const char *>(row) + (F32 ? 4 : 2) * first);
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) w[i] = from[i];
    }
    __device__ void floats(float (&y)[8]) const
    {
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                y[4 * i] = __uint_as_float(w[i].x); y[4 * i + 1] = __uint_as_float(w[i].y);
                y[4 * i + 2] = __uint_as_float(w[i].z); y[4 * i + 3] = __uint_as_float(w[i].w);
            }
        } else {
            const uint32_t v[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
        }
    }
};
// bf16 rows pass the caches by on their way out: 4096 rows of 1024 channels, two outputs, 7.0 us for 8.7, 13740 rows 18.2 for 22.2, 137400 186 for 192, 13740 tokens of 32 heads x 64 21.5 for 23.3.  Where
// the next call reads the rows at once that gains and loses nothing (both calls: 64 rows of 2048 9.9 us either way, 13740 of 1024 37.5, 4096 11.3 for 13.0).  float32 rows do not, whose two stores a lane are
// halves of a line each (16411 tokens of 40 heads x 128 134 us, 139 past the caches).
template <bool F32>
__device__ inline void store_eight(void *row, int first, const float (&y)[8])
{
    if constexpr (F32) {
        float4 *const to = reinterpret_cast<float4 *>(static_cast<float *>(row) + first);
        to[0] = make_float4(y[0], y[1], y[2], y[3]);
        to[1] = make_float4(y[4], y[5], y[6], y[7]);
    } else {
        typedef uint32_t Four __attribute__((ext_vector_type(4)));
        const Four v = {pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
        __builtin_nontemporal_store(v, reinterpret_cast<Four *>(static_cast<uint16_t *>(row) + first));
    }
}
__device__ inline void load_eight(const float *from, float (&y)[8])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float4 v = reinterpret_cast<const float4 *>(from)[i];
        y[4 * i] = v.x; y[4 * i + 1] = v.y; y[4 * i + 2] = v.z; y[4 * i + 3] = v.w;
    }
}

// 1 / sqrt(v).  The instruction takes a number below 2^-126 for 0; those, and some more, are lifted first.
__device__ inline float inverse_root(float v)
{
    const bool low = v < 0x1p-100f;
    const float r = __builtin_amdgcn_rsqf(low ? v * 0x1p100f : v);
    return low ? r * 0x1p50f : r;
}

}  // namespace qvggt

// What a block's output does to the residual stream, and the norm in front of the next block:
//     x' = x + scale gate[r] norm_post(y),      h = norm_pre(x') (1 + mod_scale[r]) + mod_shift[r].
//
// One pass: LANES lanes have a row, every one V pieces of eight channels, in registers from the first load to the last store; means and variances are two passes over registers.
#include "block_rows.h"

namespace qvggt {
namespace {

template <int LANES>
__device__ inline float row_sum(float v, float *red)
{
    if (LANES == 16) {
        v = dpp_add_step<0xB1>(v);
        v = dpp_add_step<0x4E>(v);
        v = dpp_add_step<0x141>(v);
        return dpp_add_step<0x140>(v);
    }
    v = sum_over_64_lanes(v);
    if (LANES == 64) return v;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (red[0] + red[1]) + (red[2] + red[3]);
    __syncthreads();
    return v;
}

// Norm of a row; pieces behind its end hold zeros before and anything after.
template <int LANES, int V>
__device__ inline void normalise(float (&y)[V][8], int kind, int C, float eps, int lane, float *red)
{
    if (kind == kNormNone) return;
    const float share = 1.0f / C;
    if (kind == kNormLayer) {
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += y[v][i];
        const float mean = row_sum<LANES>(s, red) * share;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) y[v][i] -= mean;
    }
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v)
        if ((v * LANES + lane) * 8 < C)
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(y[v][i], y[v][i], s);
    const float f = inverse_root(row_sum<LANES>(s, red) * share + eps);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[v][i] *= f;
}

// Eight channels of a condition's row.
__device__ inline void load_cond(const void *row, bool f32, int first, float (&u)[8])
{
    if (f32) {
        load_eight(static_cast<const float *>(row) + first, u);
    } else {
        Eight<false> raw;
        raw.load(row, first);
        raw.floats(u);
    }
}

template <int LANES, int V, bool XF, bool YF, bool HF>
__global__ __launch_bounds__(256) void residual_norm_kernel(ResidualNorm a)
{
    __shared__ float red[4];
    const int lane = threadIdx.x % LANES;
    const long long row = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    if (row >= a.M) return;
    const size_t at = (size_t)row * a.C;
    const char *const x_row = static_cast<const char *>(a.x) + at * (XF ? 4 : 2), *const y_row = static_cast<const char *>(a.y) + at * (YF ? 4 : 2);
    auto piece = [&](int v) { return (v * LANES + lane) * 8; };
    auto there = [&](int v) { return piece(v) < a.C; };
    Eight<XF> raw_x[V];
    Eight<YF> raw_y[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (there(v)) {
            raw_x[v].load(x_row, piece(v));
            if (a.y != nullptr) raw_y[v].load(y_row, piece(v));
        }
    const bool conditioned = a.gate != nullptr || a.mod_scale != nullptr || a.mod_shift != nullptr;
    const int r = !conditioned ? 0 : a.row_of != nullptr ? min(max(a.row_of[row], 0), a.cond_rows - 1) : a.cond_rows == 1 ? 0 : (int)row;
    const size_t cond = (size_t)r * a.cond_stride * (a.cond_f32 ? 4 : 2);

    float x[V][8];
    if (a.y != nullptr) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            raw_y[v].floats(x[v]);
            if (!there(v))
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] = 0.0f;
        }
        normalise<LANES, V>(x, a.post_norm, a.C, a.eps, lane, red);
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (there(v)) {
                float u[8];
                if (a.post_gain != nullptr) {
                    load_eight(a.post_gain + piece(v), u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[v][i] *= u[i];
                }
                if (a.post_bias != nullptr) {
                    load_eight(a.post_bias + piece(v), u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[v][i] += u[i];
                }
                if (a.scale != nullptr) {
                    load_eight(a.scale + piece(v), u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[v][i] *= u[i];
                }
                if (a.gate != nullptr) {
                    load_cond(static_cast<const char *>(a.gate) + cond, a.cond_f32, piece(v), u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[v][i] *= u[i];
                }
            }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float u[8];
        raw_x[v].floats(u);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[v][i] = !there(v) ? 0.0f : a.y != nullptr ? u[i] + x[v][i] : u[i];
        if (a.x_out != nullptr && there(v)) store_eight<XF>(static_cast<char *>(a.x_out) + at * (XF ? 4 : 2), piece(v), x[v]);
    }
    if (a.h == nullptr) return;
    normalise<LANES, V>(x, a.norm, a.C, a.eps, lane, red);
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (there(v)) {
            float u[8];
            if (a.gain != nullptr) {
                load_eight(a.gain + piece(v), u);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] *= u[i];
            }
            if (a.bias != nullptr) {
                load_eight(a.bias + piece(v), u);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] += u[i];
            }
            if (a.mod_scale != nullptr) {
                load_cond(static_cast<const char *>(a.mod_scale) + cond, a.cond_f32, piece(v), u);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] = fmaf(x[v][i], u[i], x[v][i]);
            }
            if (a.mod_shift != nullptr) {
                load_cond(static_cast<const char *>(a.mod_shift) + cond, a.cond_f32, piece(v), u);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] += u[i];
            }
            store_eight<HF>(static_cast<char *>(a.h) + at * (HF ? 4 : 2), piece(v), x[v]);
        }
}

template <int LANES, int V, bool XF, bool YF, bool HF>
hipError_t launch(const ResidualNorm &a, hipStream_t stream)
{
    residual_norm_kernel<LANES, V, XF, YF, HF><<<dim3((unsigned)(((long long)a.M * LANES + 255) / 256)), 256, 0, stream>>>(a);
    return hipGetLastError();
}
template <bool XF, bool YF, bool HF>
hipError_t launch(const ResidualNorm &a, hipStream_t stream)
{
    if (a.C <= 128) return launch<16, 1, XF, YF, HF>(a, stream);
    if (a.C <= 256) return launch<16, 2, XF, YF, HF>(a, stream);
    if (a.C <= 512) return launch<64, 1, XF, YF, HF>(a, stream);
    if (a.C <= 1024) return launch<64, 2, XF, YF, HF>(a, stream);
    if (a.C <= 2048) return launch<64, 4, XF, YF, HF>(a, stream);
    if (a.C <= 4096) return launch<256, 2, XF, YF, HF>(a, stream);
    return launch<256, 4, XF, YF, HF>(a, stream);
}

}  // namespace

hipError_t run_residual_norm(const ResidualNorm &a, hipStream_t stream)
{
    switch (a.x_f32 * 4 + a.y_f32 * 2 + a.h_f32) {
        case 0: return launch<false, false, false>(a, stream);
        case 1: return launch<false, false, true>(a, stream);
        case 2: return launch<false, true, false>(a, stream);
        case 3: return launch<false, true, true>(a, stream);
        case 4: return launch<true, false, false>(a, stream);
        case 5: return launch<true, false, true>(a, stream);
        case 6: return launch<true, true, false>(a, stream);
        default: return launch<true, true, true>(a, stream);
    }
}

}  // namespace qvggt

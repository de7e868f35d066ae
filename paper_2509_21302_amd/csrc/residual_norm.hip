// What a block's output does to the residual stream, and the norm in front of the next block:
//     x' = x + scale gate[r] norm_post(y),      h = norm_pre(x') (1 + mod_scale[r]) + mod_shift[r].
//
// One pass: LANES lanes have a row, every one V pieces of eight channels, in registers from the first load to the last store; means and variances are two passes over registers.  Bound by memory:
// 5.4 to 5.9 TB/s, read and written, from 128 to 8192 channels (137400 rows of 1024 in bf16: 192 us), where a copy reaches 4.7 to 5.4 by its size; 4.8 with gains, gate, scale and shift of everything, which are
// more bytes a row than the row itself, out of L2.
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
    v = 0.0f;
    for (int i = 0; i < (int)blockDim.x / 64; ++i) v += red[i];
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
        if ((v * (LANES ? LANES : 64) + lane) * 8 < C)
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(y[v][i], y[v][i], s);
    const float f = inverse_root(row_sum<LANES>(s, red) * share + eps);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[v][i] *= f;
}

// Eight channels of a row of a condition, or of a vector; what is not given is not looked at.
__device__ inline void load_cond(const void *rows, size_t at, bool f32, int first, float (&u)[8])
{
    if (rows == nullptr) return;
    const char *const row = static_cast<const char *>(rows) + at;
    if (f32) {
        load_eight(reinterpret_cast<const float *>(row) + first, u);
    } else {
        Eight<false> raw;
        raw.load(row, first);
        raw.floats(u);
    }
}
__device__ inline void load_given(const float *from, int first, float (&u)[8])
{
    if (from != nullptr) load_eight(from + first, u);
}
__device__ inline void multiply(const void *given, float (&x)[8], const float (&u)[8])
{
    if (given != nullptr)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= u[i];
}
__device__ inline void add(const void *given, float (&x)[8], const float (&u)[8])
{
    if (given != nullptr)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += u[i];
}

// LANES = 0: a block has a row, of as many lanes as it has pieces.
template <int LANES, int V, bool XF, bool YF, bool HF>
__global__ __launch_bounds__(LANES ? 256 : 1024) void residual_norm_kernel(ResidualNorm a, long long row0)
{
    constexpr int kLanes = LANES ? LANES : 64;          // (LANES = 0 has V = 1)
    __shared__ float red[16];
    const int lane = LANES ? threadIdx.x % kLanes : threadIdx.x;
    const long long row = row0 + (LANES ? (long long)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes : blockIdx.x);
    if (row >= a.M) return;
    const size_t at = (size_t)row * a.C;
    const char *const x_row = static_cast<const char *>(a.x) + at * (XF ? 4 : 2), *const y_row = static_cast<const char *>(a.y) + at * (YF ? 4 : 2);
    auto piece = [&](int v) { return (v * kLanes + lane) * 8; };
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
    // What a piece is multiplied by is loaded ahead of the sums where a lane has one piece of a wave's row (400000 rows of 128 channels: 68.9 us for 69.7).  Not where a block has the row: the registers
    // cost more waves than that gains (8191 rows of 2560 with everything given: 60 us for 49; 10000 of 8192: 171 for 125).
    constexpr bool kAhead = V == 1 && LANES != 0;
    float post_gain[8], post_bias[8], scale[8], gate[8], gain[8], bias[8], mod_scale[8], mod_shift[8];
    auto load_post = [&](int v) {
        load_given(a.post_gain, piece(v), post_gain);
        load_given(a.post_bias, piece(v), post_bias);
        load_given(a.scale, piece(v), scale);
        load_cond(a.gate, cond, a.cond_f32, piece(v), gate);
    };
    auto load_pre = [&](int v) {
        load_given(a.gain, piece(v), gain);
        load_given(a.bias, piece(v), bias);
        load_cond(a.mod_scale, cond, a.cond_f32, piece(v), mod_scale);
        load_cond(a.mod_shift, cond, a.cond_f32, piece(v), mod_shift);
    };
    if (kAhead && there(0)) {
        if (a.y != nullptr) load_post(0);
        if (a.h != nullptr) load_pre(0);
    }

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
                if (!kAhead) load_post(v);
                multiply(a.post_gain, x[v], post_gain);
                add(a.post_bias, x[v], post_bias);
                multiply(a.scale, x[v], scale);
                multiply(a.gate, x[v], gate);
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
            if (!kAhead) load_pre(v);
            multiply(a.gain, x[v], gain);
            add(a.bias, x[v], bias);
            if (a.mod_scale != nullptr)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[v][i] = fmaf(x[v][i], mod_scale[i], x[v][i]);
            add(a.mod_shift, x[v], mod_shift);
            store_eight<HF>(static_cast<char *>(a.h) + at * (HF ? 4 : 2), piece(v), x[v]);
        }
}

template <int LANES, int V, bool XF, bool YF, bool HF>
hipError_t launch(const ResidualNorm &a, hipStream_t stream)
{
    const int block = LANES ? 256 : (a.C / 8 + 63) / 64 * 64, rows = LANES ? 256 / (LANES ? LANES : 1) : 1;       // of a block
    const long long most = (1 << 30) / block * (long long)rows;             // of a launch, which has less than 2^32 threads
    for (long long row0 = 0; row0 < a.M; row0 += most) {
        const long long here = a.M - row0 < most ? a.M - row0 : most;
        residual_norm_kernel<LANES, V, XF, YF, HF><<<dim3((unsigned)((here + rows - 1) / rows)), block, 0, stream>>>(a, row0);
    }
    return hipGetLastError();
}
// Lanes by the row's length: few enough that all have work, and no more than a wave where a lane can hold its part.  50 million values in bf16, us (lanes x pieces; 0: a block):
//     128 channels   16 x 1   68      16 x 2   73     64 x 1  182         512   16 x 4   71     64 x 1   69     64 x 2   73     0   67
//     136            16 x 2   96      16 x 4  103     64 x 1  178         520   64 x 2   90     64 x 4   98     0   99
//     256            16 x 2   69      16 x 4   71     64 x 1  105        1024   64 x 2   68     64 x 4   72     0   70
//     264            16 x 4  100      64 x 1  101     0   97             1032   64 x 4   82     0   90
//     384            16 x 4   70      64 x 1   76     0   73             2048   64 x 4   71     0   72
// More pieces a lane than four cost waves: 8191 rows of 2560 channels with everything given 52 us with five, 49 with a block.
template <bool XF, bool YF, bool HF>
hipError_t launch(const ResidualNorm &a, hipStream_t stream)
{
    if (a.C <= 128) return launch<16, 1, XF, YF, HF>(a, stream);
    if (a.C <= 256) return launch<16, 2, XF, YF, HF>(a, stream);
    if (a.C <= 512) return launch<64, 1, XF, YF, HF>(a, stream);
    if (a.C <= 1024) return launch<64, 2, XF, YF, HF>(a, stream);
    if (a.C <= 2048) return launch<64, 4, XF, YF, HF>(a, stream);
    return launch<0, 1, XF, YF, HF>(a, stream);
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

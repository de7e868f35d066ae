// Attention over the 4-bit key/value cache for more rows than the waves of a block share (prompts, queries on another sequence's states): a wave has 16, 32 or 64 rows of its own and goes through all
// keys that they see; the four waves of a block go through the same pages at about the same time.
//
// What bounds it is the issue of vector and matrix instructions, of which the SIMD overlaps little: taking 4-bit words apart and exp2 on the one side, two products on the other (a prompt of
// 12289 tokens, 32 heads on 8, 128 channels: 0.82 of the cycles have a vector or matrix instruction issuing, the matrix cores are busy in 0.40; 1.32 ms, 0.94 PFLOP/s of what rows see), and, where
// a wave has four tiles, what two waves a SIMD with one step ahead wait for (1374 queries on 68700 keys, 16 heads x 64: 0.64 and 0.28 of the cycles; 0.62 ms, 0.62 PFLOP/s).  Turning tiles of codes
// into fp16 numbers in LDS once a block, so that the waves share that work, is no faster (64 keys at a time, or 32, one tile ahead: 1.30 to 1.58 ms where this was 1.27): reading them back costs what it saves.
#include "kv4_attention.h"
#include "kv4_plan.h"

namespace qvggt {
namespace {

struct Tiled {
    Kv4Attention a;
    int group, chunk, splits, tiles;    // query heads of a key head; keys of a part; parts and tiles of rows that there may be
    float *partials;                    // [seqs][heads][rows][splits][D + 2]
};
__device__ inline size_t partial_row(const Tiled &w, int b, int head, int row, int split)
{
    return (((size_t)b * w.a.pages.heads + head) * ((size_t)w.a.max_q * w.group) + row) * w.splits + split;
}

// The sequence with the place'th most keys, of every 64 of them: whichever order a batch has, the longest blocks begin first (448 queries on 1500 keys of 12 sequences at most, 20 heads x 64:
// 57.7 us in reversed and in random order, 69.3 and 72.1 without; 55 as it is now).  Not where a wave has four tiles, whose registers are full (a frame over 50: 633 us for 612) and whose blocks are many
// or of one sequence.
__device__ inline int longest(const Kv4Attention &a, int place, int lane)
{
    if (a.seqs == 1) return 0;
    const int base = place & ~63, n = min(a.seqs - base, 64), len = a.lens[base + min(lane, n - 1)];
    int before = 0;
    for (int i = 0; i < n; ++i) {
        const int other = __builtin_amdgcn_readlane(len, i);
        before += other > len || (other == len && i < lane);
    }
    return base + __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < n && before == place - base));     // (exactly one lane has it)
}

template <int D, int NT>
__global__ __launch_bounds__(256, (NT == 1 || (D == 64 && NT == 2) ? 3 : 2)) void kv4_own_rows_kernel(Tiled w)
{
    constexpr int C = D / 16, kPad = D + 4;
    __shared__ __align__(16) float area[4][16 * kPad];
    __shared__ float tops[4][16], totals[4][16], lifts[4][16 * NT];
    const Kv4Attention &a = w.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    // Heads first, parts next, then tiles from the last one on, where rows see most, sequences last: blocks that run together have keys in common (those of a head on one of the eight
    // dies, where heads are a multiple of eight), and a sequence's longest blocks begin first
    const int head = blockIdx.x % a.pages.heads, rest = blockIdx.x / a.pages.heads, place = rest % (w.tiles * w.splits);
    const int b = NT == 4 ? rest / (w.tiles * w.splits) : longest(a, rest / (w.tiles * w.splits), lane);
    const Sequence seq = sequence_of(a, b);
    const int rows = seq.n * w.group, tile = (rows + 64 * NT - 1) / (64 * NT) - 1 - place / w.splits, split = place % w.splits;
    const int row0 = (tile * 4 + wave) * 16 * NT, here = min(rows - row0, 16 * NT);
    if (tile < 0 || here <= 0) return;
    const int last = visible(a, seq, (row0 + here - 1) / w.group), full = visible(a, seq, row0 / w.group);      // keys that some row sees, and that all see
    const int t0 = split * w.chunk, stop = min(last, t0 + w.chunk);
    typedef Rows<D, NT, 1, false> Mine;
    Mine r;
    float *const mine = area[wave];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        typename Mine::Query query[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) query[k].load(a, seq, head, w.group, row0 + 16 * j + 4 * k + g, rows, lane);
#pragma unroll
        for (int k = 0; k < 4; ++k) query[k].load_angles(a, lane);
#pragma unroll
        for (int k = 0; k < 4; ++k) query[k].store(a, row0 + 16 * j + 4 * k + g < rows, mine + (4 * k + g) * kPad, lane);
        lanes_exchange_fence();
        const int row = row0 + 16 * j + (lane & 15);
        r.end[j] = row < rows ? visible(a, seq, row / w.group) : 0;
        r.take_queries(j, mine, lane);
        lanes_exchange_fence();
    }
    r.start(r.highest_exponent(), lifts[wave]);
    Keys<D, 1, false> keys;
    if (t0 < stop) keys.begin(a, b, head, last, t0, 32, lane);
    r.run(keys, t0, 32, full, last, stop, g);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        r.leave(j, mine, tops[wave], totals[wave], lane);
        lanes_exchange_fence();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r16 = 4 * k + g, row = row0 + 16 * j + r16, first = (lane & 15) * C;
            float x[C];
#pragma unroll
            for (int i = 0; i < C; ++i) x[i] = mine[r16 * kPad + first + i];
            if (row < rows) {
                if (w.splits == 1) finish_row<D>(a, w.group, seq, head, row, x, totals[wave][r16], lane);
                else leave_row<D>(w.partials + partial_row(w, b, head, row, split) * kPartial<D>, x, tops[wave][r16], totals[wave][r16], lane);
            }
        }
        lanes_exchange_fence();
    }
}

// The parts of a row put together: 16 lanes have a row.
template <int D>
__global__ __launch_bounds__(256) void kv4_join_parts_kernel(Tiled w)
{
    constexpr int C = D / 16;
    const Kv4Attention &a = w.a;
    const int lane = threadIdx.x & 63, first = (lane & 15) * C, head = blockIdx.y, b = blockIdx.z, row = blockIdx.x * 16 + (threadIdx.x >> 4);
    const Sequence seq = sequence_of(a, b);
    if (row >= seq.n * w.group) return;
    const int used = (visible(a, seq, row / w.group) + w.chunk - 1) / w.chunk;
    const float *const from = w.partials + partial_row(w, b, head, row, 0) * kPartial<D>;
    float top = kNone, total = 0.0f, x[C];
    for (int s = 0; s < used; ++s) top = fmaxf(top, from[(size_t)s * kPartial<D> + D]);
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = 0.0f;
    for (int s = 0; s < used; ++s) {
        const float *p = from + (size_t)s * kPartial<D>;
        const float f = __builtin_amdgcn_exp2f(p[D] - top);
        total = fmaf(f, p[D + 1], total);
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] = fmaf(f, p[first + i], x[i]);
    }
    finish_row<D>(a, w.group, seq, head, row, x, total, lane);
}

template <int D>
hipError_t launch(const Kv4Attention &a, hipStream_t stream)
{
    const int group = a.q_heads / a.pages.heads;
    const Kv4Tiles p = kv4_tiles(a.seqs, a.max_q, a.max_kv, a.q_heads, a.pages.heads, D);
    const Tiled w{a, group, p.chunk, p.splits, p.tiles, static_cast<float *>(a.workspace)};
    const dim3 grid((unsigned)a.seqs * a.pages.heads * p.tiles * p.splits);
    if (D == 64 && p.nt == 4) kv4_own_rows_kernel<64, 4><<<grid, 256, 0, stream>>>(w);
    else if (p.nt == 1) kv4_own_rows_kernel<D, 1><<<grid, 256, 0, stream>>>(w);
    else kv4_own_rows_kernel<D, 2><<<grid, 256, 0, stream>>>(w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    kv4_join_parts_kernel<D><<<dim3((a.max_q * group + 15) / 16, a.pages.heads, a.seqs), 256, 0, stream>>>(w);
    return hipGetLastError();
}

hipError_t run_kv4_own_rows(const Kv4Attention &a, int d, hipStream_t stream) { return d == 64 ? launch<64>(a, stream) : launch<128>(a, stream); }

}  // namespace

hipError_t run_kv4_shared_rows(const Kv4Attention &a, int d, hipStream_t stream);

size_t kv4_attention_workspace_bytes(int seqs, int max_q, int max_kv, int q_heads, int kv_heads, int d)
{
    if ((long long)max_q * (q_heads / kv_heads) <= kKv4SharedRows) return kv4_shares(seqs, max_q, max_kv, q_heads, kv_heads, d).bytes;
    return kv4_tiles(seqs, max_q, max_kv, q_heads, kv_heads, d).bytes;
}

hipError_t run_kv4_attention(const Kv4Attention &a, int d, hipStream_t stream)
{
    if ((long long)a.max_q * (a.q_heads / a.pages.heads) <= kKv4SharedRows) return run_kv4_shared_rows(a, d, stream);
    return run_kv4_own_rows(a, d, stream);
}

}  // namespace qvggt

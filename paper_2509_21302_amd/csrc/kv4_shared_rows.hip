// Attention over the 4-bit key/value cache for up to 64 rows a key head (single tokens, a few tokens): the waves of a block share the rows and take steps of 32 keys in turn.
// What bounds it is the way of the pages out of memory: one sequence of a megatoken, 8 heads x 128, 189 us, 5.86 TB/s (16 x 64: 217 us, 5.25); 64 sequences to 8192 keys, 287 MB, 60 us and
// 5 for the join.  About 10 us of a call are the way lengths, page table, pages at its start and that join.
//
// The keys of all sequences and heads, in units of a block's step, are laid end to end and cut into as many even shares as the chip holds blocks at a time: lengths of a batch may
// differ as they like, up to 512 sequences and four heads for every block that the chip holds.  A block goes through its share sequence by sequence and head by head; where a head's keys are cut, its blocks leave partial sums, at most two each, and the join
// puts them together.  Where there are few keys, or more sequences or heads than that, every head has a block of its own and nothing is joined: one sequence far longer
// than the others is what such a call waits for.
#include "kv4_attention.h"
#include "kv4_plan.h"

namespace qvggt {
namespace {

struct Shared {
    Kv4Attention a;
    int group, unit_shift;      // query heads of a key head; log2 of the keys of a unit
    int tiles, tile_rows;       // tiles of rows of a key head, and rows of one: what is said of a head below is said of each of its tiles
    int blocks, least;          // shares, and the fewest units of one; blocks = 0: a block for every head
    int32_t *map;               // [0]: units of a share, [1 + b]: what one head of all sequences before b costs
    float *partials;            // [blocks][a head that began in an earlier block, one that goes on in a later one][rows of a tile][D + 2]
};

// What a head of a sequence costs, in units: its keys (one unit at least where it has queries: a head without keys gets its zeros from a block), and in front of them what
// it takes to begin and to end with a head.
constexpr int kSetup = 2;
__device__ inline int cost_of(const Shared &w, const Sequence &s)
{
    const int units = max((s.len + (1 << w.unit_shift) - 1) >> w.unit_shift, 1) + kSetup;
    return s.n == 0 ? 0 : units;
}

// Where a unit number lies, 64 sequences at a time.  A wave keeps them in its own part of LDS (in registers they would be beside the sums).
struct Map {
    struct Place {
        int upto[64], start[64], n[64], len[64], before[64];        // cost of a head of the sequences up to and with this one; the sequence
    };
    Place *place;
    int base, before, total;            // sequences and cost before the 64; cost up to their end
    __device__ void load(const Shared &w, int first, int cost_before, int lane)
    {
        base = first;
        before = cost_before;
        const Sequence s = sequence_of(w.a, min(first + lane, w.a.seqs - 1));
        int scan = first + lane < w.a.seqs ? cost_of(w, s) : 0;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int other = __shfl_up(scan, d);
            if (lane >= d) scan += other;
        }
        lanes_exchange_fence();
        place->upto[lane] = before + scan;
        place->start[lane] = s.start;
        place->n[lane] = s.n;
        place->len[lane] = s.len;
        place->before[lane] = s.before;
        lanes_exchange_fence();
        total = before + __builtin_amdgcn_readlane(scan, 63);
    }
    // the sequence of a unit number below total * heads: its place among the 64, cost before it and up to its end
    __device__ int find(int pos, int heads, int lane, int &from, int &to) const
    {
        const int in = __builtin_ctzll(__builtin_amdgcn_ballot_w64(place->upto[lane] * heads > pos));
        to = __builtin_amdgcn_readfirstlane(place->upto[in]);
        from = in == 0 ? before : __builtin_amdgcn_readfirstlane(place->upto[max(in, 1) - 1]);
        return in;
    }
    __device__ Sequence sequence(int in) const
    {
        return {__builtin_amdgcn_readfirstlane(place->start[in]), __builtin_amdgcn_readfirstlane(place->n[in]), __builtin_amdgcn_readfirstlane(place->len[in]),
                __builtin_amdgcn_readfirstlane(place->before[in])};
    }
};

// Steps that a wave has ahead of it.  64 channels are half the bytes: two (one sequence of a megatoken, 16 heads: 214 us, 224 with one; 48 sequences to 16384 keys the same within the
// runs' spread, 90.5 and 91).  128: two take the registers of a third wave (64 sequences to 8192 keys 78 us for 69).
template <int D, int NT>
constexpr int kAhead = D == 64 && NT == 1 ? 2 : 1;

// Three waves a SIMD for 16 rows, two for 32; four for 16 rows of 64 channels leave some registers in scratch memory (48 sequences to 16384 keys, own heads: 94 us for 91).
template <int D, int NT>
__global__ __launch_bounds__(256, (NT == 1 ? 3 : 2)) void kv4_shared_rows_kernel(Shared w)
{
    constexpr int C = D / 16, kPad = D + 4;
    __shared__ __align__(16) float area[4][16 * kPad];
    __shared__ float tops[4][16], totals[4][16], lifts[4][16 * NT];
    __shared__ Map::Place places[4];
    const Kv4Attention &a = w.a;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tiles = NT == 1 ? 1 : w.tiles, heads = a.pages.heads * tiles;
    const int thread = threadIdx.x;
    Map map{&places[wave], 0, 0, 0};
    int pos = 0, stop = 1;
    if (w.blocks > 0) {
        int all = 0;
        for (int first = 0; first < a.seqs; first += 64) {
            const int lane = thread & 63;
            map.load(w, first, all, lane);
            if (blockIdx.x == 0 && wave == 0 && first + lane < a.seqs) w.map[1 + first + lane] = lane == 0 ? all : map.place->upto[lane - 1];
            all = map.total;
        }
        const int share = max((int)(((long long)all * heads + w.blocks - 1) / w.blocks), w.least);
        if (blockIdx.x == 0 && thread == 0) w.map[0] = share;
        if ((long long)blockIdx.x * share >= (long long)all * heads) return;
        pos = blockIdx.x * share;
        stop = min(pos + share, all * heads);
        if (a.seqs > 64) map.load(w, 0, 0, thread & 63);
    }
    while (pos < stop) {
        // the next head's part of the share; what the lanes' numbers lead to is worked out again for each, and not kept in registers beside the loop below
        unsigned none = 0;
        asm volatile("" : "+s"(none));
        const int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none)), g = lane >> 4;
        Sequence seq;
        int b, head, unit = 0, units = 1, part = 1;
        if (w.blocks > 0) {
            while (pos >= map.total * heads) map.load(w, map.base + 64, map.total, lane);
            int from, to;
            const int in = map.find(pos, heads, lane, from, to);
            b = map.base + in;
            seq = map.sequence(in);
            const int cost = to - from, r = pos - from * heads;
            head = r / cost;
            units = cost - kSetup;
            unit = max(r - head * cost - kSetup, 0);
            pos = from * heads + head * cost + kSetup + unit;
            part = min(units - unit, stop - pos);
            if (part <= 0) break;                           // the share ends before the head's first keys
        } else {
            b = blockIdx.x / heads;
            head = blockIdx.x - b * heads;
            seq = sequence_of(a, b);
            if (seq.n == 0) return;
        }
        const int tile = head % tiles, row0 = tile * 16 * NT, rows = seq.n * w.group;
        head /= tiles;
        if (row0 >= rows) {                     // a sequence of fewer rows
            pos += part;
            continue;
        }
        const int last = seq.len, full = visible(a, seq, row0 / w.group);
        const int t0 = (unit << w.unit_shift) + wave * 32, end = w.blocks > 0 ? min(last, (unit + part) << w.unit_shift) : last;
        Keys<D, kAhead<D, NT>, true> keys;
        if (last == 0) {                        // nothing is seen: zeros
            for (int row = row0 + 4 * wave + g; row < min(rows, row0 + 16 * NT); row += 16) {
                float x[C] = {};
                finish_row<D>(a, w.group, seq, head, row, x, 0.0f, lane);
            }
            pos += part;
            continue;
        }
        typedef Rows<D, NT, kAhead<D, NT>, true> Mine;
        typename Mine::Query query[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) query[j].load(a, seq, head, w.group, row0 + 16 * j + 4 * wave + g, rows, lane);
#pragma unroll
        for (int j = 0; j < NT; ++j) query[j].load_angles(a, lane);
        keys.begin(a, b, head, last, t0, 128, lane);                   // (a wave that has no step here fetches the last blocks)
#pragma unroll
        for (int j = 0; j < NT; ++j) query[j].store(a, row0 + 16 * j + 4 * wave + g < rows, area[j] + (4 * wave + g) * kPad, lane);
        Mine r;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int row = row0 + 16 * j + (lane & 15);
            r.end[j] = row < rows ? visible(a, seq, row / w.group) : 0;
            r.take_queries(j, area[j], lane);
        }
        r.start(r.highest_exponent(), lifts[wave]);
        r.run(keys, t0, 128, full, last, end, g);
        __syncthreads();                        // the area had the queries
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            r.leave(j, area[wave], tops[wave], totals[wave], lane);
            __syncthreads();
            const int r16 = 4 * wave + g, row = row0 + 16 * j + r16, first = (lane & 15) * C;
            const float top = fmaxf(fmaxf(tops[0][r16], tops[1][r16]), fmaxf(tops[2][r16], tops[3][r16]));
            float x[C], total = 0.0f;
#pragma unroll
            for (int i = 0; i < C; ++i) x[i] = 0.0f;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float f = __builtin_amdgcn_exp2f(tops[v][r16] - top);
                total = fmaf(f, totals[v][r16], total);
#pragma unroll
                for (int i = 0; i < C; ++i) x[i] = fmaf(f, area[v][r16 * kPad + first + i], x[i]);
            }
            if (row < rows) {
                if (part == units) finish_row<D>(a, w.group, seq, head, row, x, total, lane);
                else leave_row<D>(w.partials + ((size_t)(2 * blockIdx.x + (unit == 0)) * (16 * NT) + row - row0) * kPartial<D>, x, top, total, lane);
            }
            __syncthreads();
        }
        pos += part;
    }
}

// The shares of a row put together, where it has several: a block has a row, 16 lanes of it every sixteenth share.
template <int D>
__global__ __launch_bounds__(256) void kv4_join_shares_kernel(Shared w)
{
    constexpr int C = D / 16;
    __shared__ __align__(16) float sums[16][D + 4];
    __shared__ float tops[16], totals[16];
    const Kv4Attention &a = w.a;
    const int lane = threadIdx.x & 63, first = (lane & 15) * C, part = threadIdx.x >> 4, head = blockIdx.y, b = blockIdx.z, row = blockIdx.x;
    const int share = w.map[0], before = w.map[1 + b];
    const Sequence seq = sequence_of(a, b);
    const int cost = cost_of(w, seq), tile = row / w.tile_rows, end = before * a.pages.heads * w.tiles + (head * w.tiles + tile + 1) * cost;
    const int from = (end - cost + kSetup) / share, used = (end - 1) / share - from + 1;
    if (row >= seq.n * w.group || used == 1) return;
    float top = kNone, total = 0.0f, x[C];
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = 0.0f;
    for (int s0 = part; s0 < used; s0 += 64) {             // four shares' loads at a time
        float y[4][C];
        float2 tail[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int s = min(s0 + 16 * k, used - 1);
            const float *p = w.partials + ((size_t)(2 * (from + s) + (s == 0)) * w.tile_rows + row - tile * w.tile_rows) * kPartial<D>;
            tail[k] = *reinterpret_cast<const float2 *>(p + D);
            if (s0 + 16 * k >= used) tail[k] = make_float2(kNone, 0.0f);
#pragma unroll
            for (int i = 0; i < C / 2; ++i) {
                const float2 v = reinterpret_cast<const float2 *>(p + first)[i];
                y[k][2 * i] = v.x;
                y[k][2 * i + 1] = v.y;
            }
        }
        const float above = fmaxf(fmaxf(fmaxf(top, tail[0].x), fmaxf(tail[1].x, tail[2].x)), tail[3].x), down = __builtin_amdgcn_exp2f(top - above);
        top = above;
        total *= down;
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] *= down;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float f = s0 + 16 * k < used ? __builtin_amdgcn_exp2f(tail[k].x - above) : 0.0f;
            total = fmaf(f, tail[k].y, total);
#pragma unroll
            for (int i = 0; i < C; ++i) x[i] = fmaf(f, y[k][i], x[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i) sums[part][first + i] = x[i];
    if ((lane & 15) == 0) {
        tops[part] = top;
        totals[part] = total;
    }
    __syncthreads();
    if (part != 0) return;
    top = tops[0];
#pragma unroll
    for (int p = 1; p < 16; ++p) top = fmaxf(top, tops[p]);
    total = 0.0f;
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = 0.0f;
    for (int p = 0; p < min(used, 16); ++p) {
        const float f = __builtin_amdgcn_exp2f(tops[p] - top);
        total = fmaf(f, totals[p], total);
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] = fmaf(f, sums[p][first + i], x[i]);
    }
    finish_row<D>(a, w.group, seq, head, row, x, total, lane);
}

template <int D>
hipError_t launch(const Kv4Attention &a, hipStream_t stream)
{
    const int group = a.q_heads / a.pages.heads, rows = a.max_q * group;
    const Kv4Shares p = kv4_shares(a.seqs, a.max_q, a.max_kv, a.q_heads, a.pages.heads, D);
    Shared w{a, group, p.unit_shift, p.tiles, 16 * p.nt, p.blocks, p.least, reinterpret_cast<int32_t *>(a.workspace), reinterpret_cast<float *>(static_cast<char *>(a.workspace) + p.map_bytes)};
    const dim3 grid(p.blocks > 0 ? p.blocks : a.seqs * a.pages.heads * p.tiles);
    if (p.nt == 1) kv4_shared_rows_kernel<D, 1><<<grid, 256, 0, stream>>>(w);
    else kv4_shared_rows_kernel<D, 2><<<grid, 256, 0, stream>>>(w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.blocks == 0) return e;
    kv4_join_shares_kernel<D><<<dim3(rows, a.pages.heads, a.seqs), 256, 0, stream>>>(w);
    return hipGetLastError();
}

}  // namespace

hipError_t run_kv4_shared_rows(const Kv4Attention &a, int d, hipStream_t stream) { return d == 64 ? launch<64>(a, stream) : launch<128>(a, stream); }

}  // namespace qvggt

// How a call of qvggt_attention is cut up: arithmetic on the host, from the sizes that the caller states.
#pragma once
#include <stddef.h>

namespace qvggt {

constexpr int kAttentionTile = 32;                  // rows of a wave: query tokens times the query heads that share a key head
constexpr int kAttentionWaves = 4;
constexpr long long kAttentionMostBlocks = 1 << 23; // of a launch
constexpr int kAttentionKeys = 128;                 // parts of the keys are multiples of it

constexpr long long attention_div_up(long long a, long long b) { return (a + b - 1) / b; }

struct AttentionPlan {
    bool few;                   // the waves of a block share the rows and have keys of their own
    int tiles, chunk, splits;   // blocks of rows of a head; keys of a part, and how many of those the longest sequence has
    size_t bytes;               // of workspace
};
inline AttentionPlan attention_plan(int seqs, int max_q, int max_kv, int q_heads, int kv_heads, int d)
{
    AttentionPlan p;
    const long long rows = (long long)max_q * (q_heads / kv_heads), pairs = (long long)seqs * kv_heads;
    p.few = rows <= kAttentionTile;
    p.tiles = (int)(p.few ? 1 : attention_div_up(rows, kAttentionTile * kAttentionWaves));
    const double resident = 256 * (p.few ? 2 : d == 64 ? 3 : 2), blocks = (double)p.tiles * pairs;      // blocks that the chip holds at a time
    // Parts: turns of the resident blocks times a part's keys and what a block costs besides, and the partial sums to memory and back; in units of the time that a block takes for a key
    const double start = p.few ? 700.0 : 250.0;
    double best = 0.0;
    p.splits = 0;
    p.chunk = kAttentionKeys;
    for (int n = 1; n <= 256 && (n == 1 || (attention_div_up(max_kv, n) >= kAttentionKeys && blocks * n < 1 << 20)); ++n) {
        const int chunk = (int)(attention_div_up(attention_div_up(max_kv, n), kAttentionKeys) * kAttentionKeys);
        double turns = blocks * n / resident;
        turns = turns > 2.0 ? turns + 0.5 : (double)(int)(turns + 0.999);
        const double join = n == 1 ? 0.0 : (p.few ? 1200.0 : 200.0) + (double)pairs * rows * n * (d + 2) * 8 / 4.5e6 / 0.02;
        const double cost = turns * (chunk + start) + join;
        if (p.splits == 0 || cost < best) {
            best = cost;
            p.chunk = chunk < kAttentionKeys ? kAttentionKeys : chunk;
            p.splits = n;
        }
    }
    p.splits = max_kv > 0 ? (int)attention_div_up(max_kv, p.chunk) : 1;
    p.bytes = p.splits == 1 ? 0 : (size_t)pairs * rows * p.splits * (d + 2) * sizeof(float);
    return p;
}

}  // namespace qvggt

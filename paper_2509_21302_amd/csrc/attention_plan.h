// How a call of qvggt_attention is cut up: arithmetic on the host, from the sizes that the caller states.
#pragma once
#include <stddef.h>

namespace qvggt {

constexpr int kAttentionTile = 32;                  // rows of a wave, query tokens times the query heads that share a key head, where a block has four times as many
// Rows of a key head up to which a block's waves share them, which is what their registers hold.  32 rows that way and as many rows: 16384 keys of one sequence, 8 key heads x 128, 21.6 us and 26.5 (64 channels
// 13.7 and 20.4; 36 rows 27.7 and 21.2); 256 sequences of 256 keys 57.5 and 64.4.  The other way round where many sequences of many keys leave none to be cut: 64 of 2048 keys 125 and 102 (16 rows 111 and 102, 8 rows 101 and 103)
constexpr int kAttentionFewRows = 32;
constexpr long long kAttentionMostBlocks = 1 << 23; // of a launch
constexpr int kAttentionKeys = 128;                 // parts of the keys are multiples of it
constexpr int kAttentionMostParts = 256;            // of a sequence's keys

constexpr long long attention_div_up(long long a, long long b) { return (a + b - 1) / b; }

struct AttentionPlan {
    bool few;                   // the waves of a block share the rows and have keys of their own
    int waves;                  // of a block
    int tiles, chunk, splits;   // blocks of rows of a head; keys of a part, and how many of those the longest sequence has
    size_t bytes;               // of workspace
};
inline AttentionPlan attention_plan(int seqs, int max_q, int max_kv, int q_heads, int kv_heads, int d, int causal)
{
    AttentionPlan p;
    const long long rows = (long long)max_q * (q_heads / kv_heads), pairs = (long long)seqs * kv_heads;
    p.few = rows <= kAttentionFewRows;
    p.waves = 4;
    p.tiles = (int)(p.few ? 1 : attention_div_up(rows, kAttentionTile * 4));
    const double blocks = (double)p.tiles * pairs;
    const double most = 256.0 * (p.few ? d == 64 ? 4 : 2 : d == 64 ? 3 : 2);        // blocks that the chip holds at a time
    // Into how many parts the keys are cut, by what each number would cost, in microseconds: turns of the blocks that the chip holds, times a part's keys, and the partial sums to memory and
    // back.  Sequences are taken to have half of the keys that are stated where there are several, and causal rows to see the mean of what the first and the last one see.
    const double seen = (seqs > 1 ? 0.55 : 1.0) * max_kv, reach = !causal ? seen : max_q < max_kv ? seen - 0.5 * max_q * (seen / max_kv) : 0.5 * seen;
    double best = 0.0;
    p.splits = 0;
    p.chunk = kAttentionKeys;
    // (many rows whose blocks fill the chip are not cut: two prompts of 2048 tokens, 16 heads x 128, 46 us whole, 52 in two parts)
    const int parts = !p.few && blocks >= 0.9 * most ? 1 : kAttentionMostParts;
    for (int i = 2, n = 1; n <= parts && (n == 1 || (attention_div_up(max_kv, n) >= kAttentionKeys && blocks * n < 1 << 20)); ++i) {       // 1, 2, 3, 4, 6, 8, 12, 16, ...
        const long long chunk = attention_div_up(attention_div_up(max_kv, n), kAttentionKeys) * kAttentionKeys;
        const double live = n == 1 ? blocks : blocks * (reach / chunk + 0.5), at_once = live < most ? live : most, turns = live / at_once;
        double cost;
        if (p.few) {
            // The blocks of a CU stream 52 GB/s (64 channels: 37), all of them 5.8 TB/s; the last turn is half empty
            const double keys = n == 1 && turns > 1.0 ? reach : (double)chunk;
            const double alone = keys * (d == 64 ? 0.0069 : 0.0098) * (at_once > 256.0 ? 2 : 1), all = at_once * keys * 4 * d / 5.8e6;
            cost = (turns > 1.0 ? turns + 0.4 : 1.0) * ((alone > all ? alone + 0.15 * all : all + 0.15 * alone) + 2.5);
            if (n > 1) cost += 6.0 + 0.08 * n + live * rows * (d + 2) * 8 / 4.5e6;
        } else {
            // 64 keys: one block on a CU 0.93 us (64 channels: 0.81), two 1.63 (0.96), three 1.3.  Blocks that see different numbers of keys leave little of the last turn empty
            const double key = d == 64 ? at_once <= 256.0 ? 0.0126 : at_once <= 512.0 ? 0.0150 : 0.0203 : at_once <= 256.0 ? 0.0146 : 0.0255;
            const double all = blocks * reach * key / at_once + 0.2 * chunk * key;
            cost = 4.0 * turns + (turns > 1.0 && all > chunk * key ? all : causal && n == 1 && at_once > 256.0 ? 0.8 * chunk * key : chunk * key);
            if (n > 1) cost += 8.0 + live / p.tiles * rows * (d + 2) * 8 / 7e6;
        }
        if (p.splits == 0 || cost < best) {
            best = cost;
            p.chunk = (int)(chunk < kAttentionKeys ? kAttentionKeys : chunk);
            p.splits = n;
        }
        n = n == 1 ? 2 : i % 2 ? n / 2 * 3 : n / 3 * 4;
    }
    p.splits = max_kv > 0 ? (int)attention_div_up(max_kv, p.chunk) : 1;
    // Whole sequences of few rows, a CU for each: eight waves (one row of 32 heads on 8 x 128, 601 keys: 7.4 us, 8.3 with four; 16 heads x 64 5.6 and 6.4; as fast where keys are cut or blocks share CUs)
    if (p.few && p.splits == 1 && blocks <= 256.0) p.waves = 8;
    p.bytes = p.splits == 1 ? 0 : (size_t)pairs * rows * p.splits * (d + 2) * sizeof(float);
    return p;
}

// What either kind of call needs (a caller asks for its sizes, not for the mask).
inline size_t attention_workspace(int seqs, int max_q, int max_kv, int q_heads, int kv_heads, int d)
{
    const size_t whole = attention_plan(seqs, max_q, max_kv, q_heads, kv_heads, d, 0).bytes, causal = attention_plan(seqs, max_q, max_kv, q_heads, kv_heads, d, 1).bytes;
    return whole > causal ? whole : causal;
}

}  // namespace qvggt

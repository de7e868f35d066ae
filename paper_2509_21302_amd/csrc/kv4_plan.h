// How a call of qvggt_kv4_attention is cut up: arithmetic on the host, from the sizes that the caller states.
#pragma once
#include <stddef.h>

namespace qvggt {

constexpr long long kv4_div_up(long long a, long long b) { return (a + b - 1) / b; }

// The most blocks of 64 rows that a call may have (a launch has less than 2^32 threads).
constexpr long long kKv4MostBlocks = 1 << 23;
constexpr int kKv4SharedRows = 64;          // rows of a key head (query tokens times query heads of it) up to which a block's waves share them

// ---- shared rows: every block an even share of all keys
struct Kv4Shares {
    int nt, tiles;              // tiles of 16 rows a block takes at a time, and how often that is a head's rows
    int blocks;                 // 0: a block for every head of every sequence, nothing to join
    int unit_shift, least;      // log2 of the keys of a unit; units of a share at least
    size_t map_bytes, bytes;    // workspace: the map of units, all of it
};
inline Kv4Shares kv4_shares(int seqs, int max_q, int max_kv, int q_heads, int kv_heads, int d)
{
    // Two tiles at most: four take the registers of two waves (64 rows on 16384 keys of 16 sequences, 128 channels: 154 us, where 32 rows are 60)
    const int rows = max_q * (q_heads / kv_heads);
    Kv4Shares p{rows <= 16 ? 1 : 2, (rows + 31) / 32, 0, 7, 4, 0, 0};
    const int resident = 256 * (p.nt == 1 ? 3 : 2);           // blocks that the chip's registers hold at a time
    const long long segments = (long long)seqs * kv_heads * p.tiles;
    while (segments * (kv4_div_up(max_kv, 1LL << p.unit_shift) + 4) >= 1LL << 30) ++p.unit_shift;
    const long long units = segments * kv4_div_up(max_kv, 1LL << p.unit_shift);
    // Whole heads: where even the longest is not worth a join, where the blocks are many enough to even out by themselves as long as lengths are alike, and where every block would go through
    // more lengths than it has keys' worth of time for
    if (max_kv <= 1024 || segments >= 4 * resident || seqs > 512) return p;
    const long long blocks = kv4_div_up(units, p.least);
    p.blocks = (int)(blocks < resident ? blocks : resident);
    p.map_bytes = (size_t)kv4_div_up(4LL * (1 + seqs), 256) * 256;
    p.bytes = p.map_bytes + (size_t)p.blocks * 2 * (16 * p.nt) * (d + 2) * sizeof(float);
    return p;
}

// ---- a wave's own rows: blocks of 64 NT rows, over a part of the keys each where there are few blocks
struct Kv4Tiles {
    int nt;                     // tiles of 16 rows a wave has
    int tiles, chunk, splits;   // blocks of rows; keys of a part, and how many of those the longest sequence has
    size_t bytes;
};
inline Kv4Tiles kv4_tiles(int seqs, int max_q, int max_kv, int q_heads, int kv_heads, int d)
{
    Kv4Tiles p;
    const long long rows = (long long)max_q * (q_heads / kv_heads), pairs = (long long)seqs * kv_heads;
    // 64 channels: four tiles take a key apart half as often as two (a frame over 50: 638 us for 697), but two have half the blocks' length to even out (448 queries on 1500 keys
    // of 12 sequences: 58 us for 83).  128 channels: the registers hold two
    const bool fits = 8 * kv4_div_up(rows, 256) * 256 <= 9 * kv4_div_up(rows, 128) * 128;       // few rows more than there are
    p.nt = d == 64 && fits && (max_kv >= 8192 || kv4_div_up(rows, 256) * pairs >= 2048) ? 4 : 2;
    p.tiles = (int)kv4_div_up(rows, 64 * p.nt);
    const int resident = 256 * (p.nt == 2 && d == 64 ? 3 : 2);          // blocks that the chip's registers hold at a time
    const double blocks = (double)p.tiles * pairs;
    // How many parts: turns of the resident blocks times a part's keys and what a block costs besides, and the partial sums to memory and back; in units of a key's 40 ns
    constexpr int kLeast = 128, kMostSplits = 32;
    // A part has 2^20 keys at most as long as there may be more of them: a wave adds its keys' weights and values up in fp32, two additions every 32 keys, and the last bit of a sum of 2^16
    // terms is within 2^-9 of it in the worst case, in which every addition is rounded the same way
    constexpr int kMostKeys = 1 << 20;
    double best = 0.0;
    p.splits = 0;
    for (int n = 1; n <= kMostSplits && (n == 1 || (kv4_div_up(max_kv, n) >= kLeast && blocks * n < 1 << 20)); ++n) {
        const int chunk = (int)(kv4_div_up(kv4_div_up(max_kv, n), kLeast) * kLeast);
        double turns = blocks * n / resident;
        turns = turns > 2.0 ? turns + 0.5 : (double)(int)(turns + 0.999);
        const double join = n == 1 ? 0.0 : 200.0 + (double)pairs * rows * n * (d + 2) * 8 / 4.5e6 / 0.04;
        const double cost = turns * (chunk + 300) + join;
        if (p.splits == 0 || cost < best || p.chunk > kMostKeys) {
            best = cost;
            p.chunk = chunk < kLeast ? kLeast : chunk;
            p.splits = n;
        }
    }
    // One tile a wave: blocks of 64 rows that take 0.7 or 0.75 of the time while there are few of them, whole sequences only, where that is less (a prompt of 512 tokens, 32 heads on 8:
    // 17 us for 24 with 64 channels, 22 for 31 with 128; but a prompt of 12289 tokens 1.61 ms for 1.29)
    const double short_turns = (double)(kv4_div_up(rows, 64) * pairs) / (256 * 3);
    if (max_kv <= kMostKeys && short_turns <= 3.0 && (short_turns > 2.0 ? short_turns + 0.5 : (double)(int)(short_turns + 0.999)) * (max_kv + 300) * (d == 64 ? 0.75 : 0.7) < best) {
        p.nt = 1;
        p.tiles = (int)kv4_div_up(rows, 64);
        p.chunk = max_kv < kLeast ? kLeast : max_kv;
    }
    p.splits = max_kv > 0 ? (int)kv4_div_up(max_kv, p.chunk) : 1;
    p.bytes = p.splits == 1 ? 0 : (size_t)seqs * q_heads * max_q * p.splits * (d + 2) * sizeof(float);
    return p;
}

}  // namespace qvggt

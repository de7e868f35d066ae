// How a call of qvggt_kv4_attention is cut up: arithmetic on the host, from the sizes that the caller states.
#pragma once
#include <stddef.h>

namespace qvggt {

constexpr long long kv4_div_up(long long a, long long b) { return (a + b - 1) / b; }

constexpr int kKv4SharedRows = 64;          // rows of a key head (query tokens times query heads of it) up to which a block's waves share them

// ---- shared rows: every block an even share of all keys
struct Kv4Shares {
    int blocks;                 // 0: a block for every head of every sequence, nothing to join
    int unit_shift, least;      // log2 of the keys of a unit; units of a share at least
    size_t map_bytes, bytes;    // workspace: the map of units, all of it
};
inline Kv4Shares kv4_shares(int seqs, int max_q, int max_kv, int q_heads, int kv_heads, int d)
{
    const int rows = max_q * (q_heads / kv_heads), tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const int resident = 256 * (tiles == 1 ? (d == 64 ? 4 : 3) : tiles == 2 ? 2 : 1);           // blocks that the chip's registers hold at a time
    const long long segments = (long long)seqs * kv_heads;
    Kv4Shares p{0, 7, 4, 0, 0};
    while (segments * (kv4_div_up(max_kv, 1LL << p.unit_shift) + 4) >= 1LL << 30) ++p.unit_shift;
    const long long units = segments * kv4_div_up(max_kv, 1LL << p.unit_shift);
    // Whole heads: where even the longest is not worth a join, and where the blocks are many enough to even out by themselves
    if (max_kv <= 1024 || segments >= 4 * resident) return p;
    const long long blocks = kv4_div_up(units, p.least);
    p.blocks = (int)(blocks < resident ? blocks : resident);
    p.map_bytes = (size_t)kv4_div_up(4LL * (1 + seqs), 256) * 256;
    p.bytes = p.map_bytes + (size_t)p.blocks * 2 * rows * (d + 2) * sizeof(float);
    return p;
}

// ---- a wave's own rows: blocks of 64 NT rows, over a part of the keys each where there are few blocks
struct Kv4Tiles {
    int tiles, chunk, splits;   // blocks of rows; keys of a part, and how many of those the longest sequence has
    size_t bytes;
};
inline Kv4Tiles kv4_tiles(int seqs, int max_q, int max_kv, int q_heads, int kv_heads, int d, int rows_of_block)
{
    Kv4Tiles p;
    p.tiles = (int)kv4_div_up((long long)max_q * (q_heads / kv_heads), rows_of_block);
    const long long blocks = (long long)p.tiles * kv_heads * seqs;
    constexpr int kLeast = 512;
    long long splits = blocks > 0 ? 1024 / blocks : 1;
    const long long most = kv4_div_up(max_kv, kLeast);
    splits = splits > most ? most : splits;
    splits = splits < 1 ? 1 : splits;
    p.chunk = (int)(kv4_div_up(kv4_div_up(max_kv, splits), kLeast) * kLeast);
    p.chunk = p.chunk < kLeast ? kLeast : p.chunk;
    p.splits = (int)kv4_div_up(max_kv, p.chunk);
    p.splits = p.splits < 1 ? 1 : p.splits;
    p.bytes = p.splits == 1 ? 0 : (size_t)seqs * q_heads * max_q * p.splits * (d + 2) * sizeof(float);
    return p;
}

}  // namespace qvggt

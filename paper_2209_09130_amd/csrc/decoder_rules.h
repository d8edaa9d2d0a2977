// Which kernels the 8-bit decoder's projection and cache run.  Host arithmetic on sizes and nothing else, so that the rules can be read and tested on
// their own.
#pragma once

namespace samp {

// ---- projection of up to sixteen rows ----------------------------------------------------------------
// K is split over eight waves, sixteen blocks of 64 a wave at most (kernels for two, four, eight and sixteen).
constexpr int FEW_WAVES = 8, FEW_ROWS = 16, FEW_K = 16 * 64 * FEW_WAVES;
inline bool tokens_few(int M, int K) { return M <= FEW_ROWS && K <= FEW_K; }
inline int tokens_few_blocks(int K)
{
    const int blocks = (K / 64 + FEW_WAVES - 1) / FEW_WAVES;
    return blocks <= 2 ? 2 : blocks <= 4 ? 4 : blocks <= 8 ? 8 : 16;
}
// With the quantiser in the same launch, which saves one, or in front.  Every block (16 channels) reads and quantises all rows: one round of its waves for up to eight rows,
// two for more, which only pays where rows are short and blocks are no more than one for each CU; and a row of more than 4096 values takes so many registers that a
// CU holds one block.  us in a chain of launches, weights from memory, K x N, one launch / two: 4096 x 4096 1 row 6.1 / 6.9, 8 7.0 / 7.4, 12 7.9 / 7.7; 4096 x 8192 1 9.0 / 9.4,
// 8 9.9 / 10.1, 12 11.3 / 10.8; 3328 x 6144 8 8.5 / 8.7, 16 11.3 / 10.1; 2048 x 4096 12 5.4 / 5.9, 16 5.9 / 6.1; 2048 x 8192 12 7.4 / 7.3, 16 8.2 / 7.6;
// 5120 x 4096 1 7.9 / 7.9, 8 8.6 / 8.6, 9 9.8 / 8.7; 5120 x 5120 1 12.7 / 10.8, 8 14.2 / 12.6; 8192 x 2048 1 7.5 / 7.8, 6 8.9 / 8.6; 8192 x 8192 1 18.4 / 16.3.  (Alone, from
// the host, the second launch costs another 3 us, so a draw goes to one.)  The codes have to leave a block below 64 KB of LDS.
constexpr int FEW_CODES = 54 << 10;
inline bool tokens_fused(int M, int N, int K)
{
    return tokens_few(M, K) && M * (K + 16) <= FEW_CODES && (M <= 8 ? K <= 4096 || N <= 4096 : K <= 2048 && N <= 4096);
}
inline bool tokens_fused_any(int M, int K) { return tokens_fused(M, 1 << 30, K); }           // for every N

// ---- projection of more rows -------------------------------------------------------------------------
// The tile (16 mt rows, 64 ntw channels) whose cost is least: its time for K = 4096 where the chip is full of it (small ones: where it is not), times the rounds of blocks
// (the mean of whole rounds and their fraction).  Over 36 random shapes (17 to 16384 rows, K 256 to 8192, N 256 to 8192) the choice costs 4 % on average against the best
// of eleven tiles and depths.  us, M x N x K, the tiles in the order of the list: 64 x 4096 x 4096 7.5 / 8.1 / 11.8 / 16.3 / 21.7; 512 x 4096 x 4096 39 / 15.5 /
// 13.1 / 17.1 / 22.5; 2048 x 4096 x 4096 148 / 76 / 73 / 34 / 39; 8192 x 4096 x 4096 583 / 296 / 290 / 129 / 126; 4096 x 11008 x 4096 781 / 396 / 400 / 188 / 181.
// What bounds the large ones is how fast a CU gets its operands from L2: a stage of 128 bytes of K is 32 KB (8 x 2) or 40 KB (8 x 3) for 512 and 768 clocks of matrix
// work, 62 and 52 bytes per clock.
struct TokensTile { int mt, ntw; float us; };
constexpr TokensTile TOKENS_TILES[] = {{2, 1, 7.3f}, {4, 1, 7.8f}, {4, 2, 13.0f}, {8, 2, 17.0f}, {8, 3, 23.0f}};
inline int tokens_tile(int M, int N)
{
    int best = 0;
    float least = 0.0f;
    for (int i = 0; i < 5; i++) {
        const long bm = 16 * TOKENS_TILES[i].mt, bn = 64 * TOKENS_TILES[i].ntw, blocks = (M + bm - 1) / bm * ((N + bn - 1) / bn);
        const float rounds = blocks <= 256 ? 1.0f : 0.5f * ((float)((blocks + 255) / 256) + (float)blocks / 256.0f), cost = rounds * TOKENS_TILES[i].us;
        if (i == 0 || cost < least) { best = i; least = cost; }
    }
    return best;
}
// Stages in flight.  Four instead of two (64 x 4096 x 4096 7.5 / 9.7) where no more is left over for it, and always on the smallest tile (85 x 1312 x 8064 12.3 / 17.2;
// 619 x 2624 x 3328 on 4 x 2 tiles, 256 left over, 14.0 / 12.3)
inline int tokens_depth(int tile, int K) { return tile <= 2 && K >= 512 && (tile == 0 || K % 512 < 256) ? 4 : 2; }
// Row tiles of a band: 2048 x 4096 x 4096 on 8 x 2 tiles, one row tile a band / eight 41.6 / 33.8, 8192 x 4096 x 4096 on 8 x 3, one / four / eight 139 / 126 / 136.
inline int tokens_band(int tile) { return tile == 4 ? 4 : 8; }

// ---- cache -------------------------------------------------------------------------------------------
// Four rows a lane group where there are blocks enough: one / four, 16 prompts of 900 to 2048 tokens written 36.2 / 33.3 us, read 31.0 / 25.3; a chunk of 4 x 512 tokens
// has 2048 x 8 rows and is better off with one (5.4 us).
inline int cache_passes(long rows, int kv_heads) { return rows * kv_heads >= 32768 ? 4 : 1; }

}  // namespace samp

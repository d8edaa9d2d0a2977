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

// ---- beam search's selection -----------------------------------------------------------------------------
// A row is cut into pieces of 512 threads with eight vectors of 16 bytes each where that makes enough of them, else of 256 with two.  us, both kernels, long / short pieces, rows x vocabulary:
// 16 bits 64 x 32000 14.0 / 10.8, 256 x 32000 14.3 / 14.0, 512 x 32000 17.8 / 18.9, 64 x 128256 13.6 / 14.3, 128 x 128256 16.9 / 19.5; binary32, whose short pieces are half as many
// values, 4 x 21128 11.9 / 9.6, 64 x 32000 12.0 / 11.3, 16 x 128256 12.0 / 12.8, 32 x 128256 12.3 / 14.3, 512 x 32000 20.6 / 25.2, 128 x 128256 20.9 / 26.4.
// A long piece takes as long as five or six short ones, full or not: 16 bits 1024 x 1000 21.4 / 13.4, 1024 x 16000 21.7 / 19.2, 1024 x 21000 23.0 / 23.3, 1024 x 36000 30.8 / 29.8, 1024 x 50304
// 31.5 / 38.6; binary32 1024 x 8000 18.4 / 17.4, 1024 x 12000 19.9 / 21.5, 512 x 12000 15.4 / 15.1, 512 x 21000 18.6 / 20.2.  Around the border the other kind is up to 0.7 us faster (64 x 128256 of
// 16 bits goes to the short ones, 64 x 32000 and 512 x 12000 of binary32 to the long ones).
struct BeamPiece { int threads, vectors; };
constexpr BeamPiece LONG_PIECE{512, 8}, SHORT_PIECE{256, 2};
inline int piece_chunks(BeamPiece p, bool wide, int vocab)
{
    const int vector = wide ? 4 : 8, values = p.threads * p.vectors * vector;
    return (vocab + vector - 1 + values - 1) / values;                // (room for `vector` - 1 values more than a row has: a piece of those alone is empty)
}
inline bool long_pieces(bool wide, int rows, int vocab)
{
    const int chunks = piece_chunks(LONG_PIECE, wide, vocab);
    return (long)rows * chunks >= (wide ? 128 : 512) && 2 * piece_chunks(SHORT_PIECE, wide, vocab) >= 11 * chunks;
}

// A launch has fewer than 2^32 threads in a direction
constexpr long LAUNCH_THREADS = 1l << 32;
inline bool pieces_fit(bool wide, long rows, int vocab)
{
    const BeamPiece p = rows < 1l << 31 && long_pieces(wide, (int)rows, vocab) ? LONG_PIECE : SHORT_PIECE;
    return rows * piece_chunks(p, wide, vocab) * p.threads < LAUNCH_THREADS;
}

// ---- bookkeeping of pages ------------------------------------------------------------------------------
// One block does a whole call where its counters fit the LDS of a CU (two of 4 bytes for each page and a list of 2, a plan of 32 bytes and a number for each new row and 16 bytes for each
// old one; 6 bytes for each page) and its 16 waves are, called from the host, no slower than the launches of several, four more of which cost another 10 us there.  In a recorded graph they are, by up to a quarter, near the border:
// us in a chain of recorded calls, one block / several kernels: pages forked, pages x rows x width, 300 x 4 x 20 5.4 / 13.6,
// 4000 x 256 x 40 9.6 / 15.6, 14000 x 64 x 64 13.8 / 15.7, 13000 x 256 x 64 16.7 / 15.6, 12000 x 64 x 512 17.3 / 15.4, 6000 x 1024 x 32 21.1 / 16.8, 9000 x 1024 x 64 28.4 / 17.3
// compacted, pages, 300 2.9 / 8.2,
// 4096 4.9 / 10.2, 8192 10.9 / 11.3, 16384 24.8 / 13.9.
inline long fork_block_lds(long pages, long rows_from, long rows) { return 10 * ((pages + 3) & ~3l) + 16 * rows_from + (32 + 4) * rows; }
inline bool fork_in_block(long pages, long rows_from, long width, long rows) { return fork_block_lds(pages, rows_from, rows) <= 150 << 10 && rows_from * width <= 32768; }
inline long compact_block_lds(long pages) { return 4 * pages + 2 * (pages / 2 + 1); }
inline bool compact_in_block(long pages, long entries) { return pages <= 8192 && entries <= 65536; }

// ---- pages that are read -------------------------------------------------------------------------------
// The scores of up to 256 pages of a sequence (64 a wave) are formed by the block that chooses among them, those of more in a launch of their own: one CU gets 35 to 50 GB/s of bounds from
// pages all over memory.  us, one launch / two: sequences x key heads x pages 1 x 8 x 256 7.4 / 9.0, 8 x 8 x 100 5.8 / 8.5, 64 x 8 x 128 7.7 / 10.6, 64 x 8 x 256 11.7 / 12.8; a
// block of sixteen waves for 1 x 8 x 1563 21 / 11.
constexpr int SCORED_TOGETHER = 256;
inline bool scores_apart(int width) { return width > SCORED_TOGETHER; }
// Threads of a block that chooses among scores that are there, by the most pages that it can have.  us, scores and choice, with 256 / 512 / 1024, sequences x 8 key heads x pages: 1 x 300 8.1 / 7.8 / 8.2,
// 64 x 512 20.3 / 20.4 / 21.6, 1 x 1000 9.2 / 8.4 / 8.9, 64 x 1000 34.6 / 34.2 / 35.0, 1 x 1563 11.0 / 9.2 / 9.1, 32 x 1563 30.6 / 28.1 / 28.2, 1 x 4000 15.4 / 11.7 / 10.4, 1 x 32768 84 / 54 / 42
inline int choice_threads(int width) { return width <= 512 ? 256 : width <= 1024 ? 512 : 1024; }
// Of the two launches that of the scores, 256 threads for each 128 pages of a sequence and a key head, always has more threads
constexpr int SCORES_BLOCK = 128;
inline bool choice_fits(long batch, long kv_heads, int width)
{
    return batch * kv_heads * (scores_apart(width) ? (width + SCORES_BLOCK - 1) / SCORES_BLOCK : 1) * 256 < LAUNCH_THREADS;
}

}  // namespace samp

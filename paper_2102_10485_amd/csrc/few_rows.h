// Rules for products of few rows (group_product.h) on what the host knows of a call: the rows of an expert on average, not the offsets.  Plain arithmetic, which the host can test.
#pragma once

namespace gan {

// Sixteens of rows, one or two, of the rows' gradient in fp32 of experts with `each` rows on average, sums of k, and `blocks` blocks if they take 32 rows.  Two read the weights once for twice the
// rows, in blocks of which a CU has one at a time where it has two of the others: they win from so many blocks on that the others, twice as many, no longer run together, of the shortest sums (k is 512 at
// least: shorter ones of more than eight rows go to tiles) from fewer.  us by 16 rows, by 32, in brackets with an epilogue: two experts of 92 rows, 1856 <- 512 (232 blocks) 12.5, 9.1 (13.1, 9.6); one of
// 1000, 512 <- 512 (264) 9.1, 8.3 (10.0, 8.9); ten of 112, 784 <- 512 (585) 23.9, 18.8 (26.3, 19.9); 50 of 30, 784 <- 512 (1261) 39.6, 30.7 (40.6, 32.4); a hundred of 24, 1024 <- 1024 (2816) 108, 96
// (112, 98).  But two of 100, 512 <- 512 (72) 6.0, 8.3 (6.6, 8.9); one of 300, 256 <- 512 (44) 6.0, 8.1 (6.7, 8.6); 17 of 48, 512 <- 1094 (344) 16.6, 24.7 (17.0, 25.6); 16 of 25, 1024 <- 2048 (464)
// 40.4, 43.9 (43.4, 45.7).  Over 620 drawn sizes, in time by 16 rows alone: 0.95 (0.93) on average, at worst 1.23 (1.14), where the blocks are a few more than whole turns of the CUs: 51 of 67, 256 <- 513
// (636) 18.6, 22.9; 64 of 20, 512 <- 512 (840) 19.4, 22.5 (21.1, 23.0).
inline int dgrad_sixteens(long long each, long long blocks, int k) { return each > 16 && blocks >= (k <= 576 ? 160 : 512) ? 2 : 1; }

// Whether two sets of waves share the sums of 8-bit tiles with an epilogue beyond 256 tiles by launch_large's count, which adds one for every expert's last rows.  Experts of up to 64 rows have one tile,
// of half the height mostly, for each of `cols` columns of tiles.  Two sets leave room for one block a CU, and win where every tile has a CU of its own and the sum is long (the two heights are dealt to
// the eight XCDs apart, so that columns that are no multiple of eight may cost each a block more).  us by one set, by two: eight experts of 32 rows, 4096 -> 4096 (256 tiles) 37.8, 34.7, of 62 44.6,
// 41.7; four of 37, 4096 -> 7936 (248) 36.1, 31.9; 16 of 40, 4096 -> 2048 (256) 36.9, 36.2; 32 of 20, 2048 -> 1024 (256) 21.2, 20.3.  But eight of 32, 1024 -> 4096 (256) 14.6, 15.1; 64 of 60,
// 2048 -> 512 (256 in four columns) 31.6, 37.2; 16 of 32, 2048 -> 2176 (272) 28.8, 35.5; 64 of 40, 1024 -> 768 (384) 20.1, 27.4; a hundred of 16, 1024 -> 1024 (800) 36.5, 51.7; and one that this
// rule takes wrongly, 32 of 40, 4096 -> 1024 (256) 37.2, 40.6.  Over 110 drawn sizes of 257 to 620 by the count, in time by one set alone: 0.99, at worst 1.01.
inline bool two_sets8(long long each, long long groups, long long cols, int k) { return each <= 64 && k >= 2048 && groups * cols <= (cols % 8 ? 248 : 256); }

}  // namespace gan

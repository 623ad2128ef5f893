// How many rows a block of the fp32 gradient for few rows takes (group_product.h).  Plain arithmetic, which the host can test.
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

}  // namespace gan

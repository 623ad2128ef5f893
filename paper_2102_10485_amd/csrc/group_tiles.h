// Which expert a tile of rows belongs to.  Every wave finds it from the offsets on its own: 64 experts at a time, a lane each, with a running maximum
// (offsets that decrease or lie outside the rows are taken as the nearest that do not) and a running sum of tiles.
#pragma once

#include "common.h"

namespace gan {

__device__ __forceinline__ int wave_scan_max(int v) {
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(v, d);
    v = l >= d ? max(v, o) : v;
  }
  return v;
}
__device__ __forceinline__ int wave_scan_add(int v) {
  const int l = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(v, d);
    v += l >= d ? o : 0;
  }
  return v;
}

// The t-th tile of `height` rows, counted expert by expert: its expert (`groups` for rows behind the last offset), its first row, and the end of the expert's
// rows.  False where there are fewer tiles.  All 64 lanes of a wave call it.
__device__ __forceinline__ bool find_tile(const int* offs, int groups, int rows, int height, unsigned t, int& group, int& row, int& end) {
  const int l = threadIdx.x & 63;
  int done = 0;                                                   // rows of the experts before
  unsigned before = 0;                                            // and their tiles
  for (int g0 = 0; g0 <= groups; g0 += 64) {
    const int g = g0 + l;
    int hi = g < groups ? min(max(offs[g + 1], 0), rows) : rows;
    hi = max(wave_scan_max(hi), done);
    int lo = __shfl_up(hi, 1);
    if (l == 0) lo = done;
    const unsigned tiles = ((unsigned)(hi - lo) + height - 1) / height;
    const unsigned upto = before + (unsigned)wave_scan_add((int)tiles);
    const unsigned long long past = __ballot(upto > t);
    if (past) {
      const int src = __ffsll((unsigned long long)past) - 1;
      const unsigned first = (unsigned)__shfl((int)(upto - tiles), src);
      group = __builtin_amdgcn_readfirstlane(g0 + src);
      row = __builtin_amdgcn_readfirstlane(__shfl(lo, src) + (int)(t - first) * height);
      end = __builtin_amdgcn_readfirstlane(__shfl(hi, src));
      return true;
    }
    done = __shfl(hi, 63);
    before = (unsigned)__shfl((int)upto, 63);
  }
  return false;
}

// Tiles of `height` rows: whole ones, and each expert's shorter last one: of more than height / 2 rows (HIGH), more than height / 4 (HALF), or fewer.
enum TileSort { WHOLE, HIGH, HALF, LOW, SORTS };

__device__ __forceinline__ unsigned tiles_of(int sort, unsigned rows, unsigned height) {
  const unsigned rest = rows % height;
  return sort == WHOLE ? rows / height : sort == HIGH ? rest > height / 2 : sort == HALF ? rest > height / 4 && rest <= height / 2 : rest > 0 && rest <= height / 4;
}

// How many of each there are.  All 64 lanes of a wave call it.
__device__ __forceinline__ void count_tiles(const int* offs, int groups, int rows, int height, unsigned (&count)[SORTS]) {
  const int l = threadIdx.x & 63;
  int done = 0;
#pragma unroll
  for (int s = 0; s < SORTS; ++s) count[s] = 0;                   // (this lane's)
  for (int g0 = 0; g0 <= groups; g0 += 64) {
    const int g = g0 + l;
    int hi = g < groups ? min(max(offs[g + 1], 0), rows) : rows;
    hi = max(wave_scan_max(hi), done);
    int lo = __shfl_up(hi, 1);
    if (l == 0) lo = done;
#pragma unroll
    for (int s = 0; s < SORTS; ++s) count[s] += tiles_of(s, (unsigned)(hi - lo), height);
    done = __shfl(hi, 63);
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2)
#pragma unroll
    for (int s = 0; s < SORTS; ++s) count[s] += (unsigned)__shfl_xor((int)count[s], d);
#pragma unroll
  for (int s = 0; s < SORTS; ++s) count[s] = (unsigned)__builtin_amdgcn_readfirstlane((int)count[s]);
}

// The t-th tile of a sort: its expert (`groups`: rows of none), its first row, and the end of the expert's rows.
__device__ __forceinline__ void find_tile_of(int sort, const int* offs, int groups, int rows, int height, unsigned t, int& group, int& row, int& end) {
  const int l = threadIdx.x & 63;
  int done = 0;
  unsigned before = 0;
  for (int g0 = 0; g0 <= groups; g0 += 64) {
    const int g = g0 + l;
    int hi = g < groups ? min(max(offs[g + 1], 0), rows) : rows;
    hi = max(wave_scan_max(hi), done);
    int lo = __shfl_up(hi, 1);
    if (l == 0) lo = done;
    const unsigned n = (unsigned)(hi - lo), tiles = tiles_of(sort, n, height);
    const unsigned upto = before + (unsigned)wave_scan_add((int)tiles);
    const unsigned long long past = __ballot(upto > t);
    if (past) {
      const int src = __ffsll((unsigned long long)past) - 1;
      const unsigned at = sort == WHOLE ? t - (upto - tiles) : n / height;
      group = __builtin_amdgcn_readfirstlane(g0 + src);
      row = __builtin_amdgcn_readfirstlane(__shfl(lo + (int)at * height, src));
      end = __builtin_amdgcn_readfirstlane(__shfl(hi, src));
      return;
    }
    done = __shfl(hi, 63);
    before = (unsigned)__shfl((int)upto, 63);
  }
}

// the rows of one expert
__device__ __forceinline__ void group_rows(const int* offs, int groups, int rows, int group, int& begin, int& end) {
  const int l = threadIdx.x & 63;
  int done = 0;
  for (int g0 = 0;; g0 += 64) {
    const int g = g0 + l;
    int hi = g < groups ? min(max(offs[g + 1], 0), rows) : rows;
    hi = max(wave_scan_max(hi), done);
    int lo = __shfl_up(hi, 1);
    if (l == 0) lo = done;
    if (group < g0 + 64) {
      begin = __builtin_amdgcn_readfirstlane(__shfl(lo, group - g0));
      end = __builtin_amdgcn_readfirstlane(__shfl(hi, group - g0));
      return;
    }
    done = __shfl(hi, 63);
  }
}

// the most tiles that `rows` rows of `groups` experts make, those of no expert among them
inline long long most_tiles(long long rows, long long groups, int height) {
  const long long with_rows = groups + 1 < rows ? groups + 1 : rows;
  return rows / height + with_rows;
}

}  // namespace gan

// The gradient through the activation behind a product grouped by label, with the bias's gradient on the way.
//
//   dz = dy act'(z),    dbias[g] = sum of dz over g's rows
//
// Bound by memory, one pass over dy and z.  Blocks take tiles of rows of one expert each and 128 columns, and leave the sums of their rows, which a second kernel adds up
// expert by expert, in order.
#include "activation.h"
#include "group_tiles.h"

#include <algorithm>

namespace gan {
namespace {

struct ActBackArgs {
  const void *dy, *z;
  const int* offs;
  void* dz;
  float* partial;                                                 // [tiles][cols], or NULL
  long long dy_stride, z_stride, dz_stride;
  int groups, rows, cols, act;
  int tall;                                                       // rows of a tile
  long long tiles;                                                // of rows, at most
};

// Tiles of 128 rows and 128 columns, of 32 rows where those would leave CUs idle.  A wave then reads 256 bytes of each of four rows at a time, and the blocks that run together whole rows
// (bf16, 16384 x 4096 of eight experts with both launches: 83 us = 4.9 TB/s; 1 KiB of a row by a wave 95; results through the caches 87; operands converted as they arrive, two waves a SIMD 157;
// ten experts' 1117 rows of 512 in fp32 7.9).
constexpr int LANES = 16, WIDE = LANES * 8, AT = 256 / LANES;     // lanes of a row, columns of a tile, its rows at a time
// Up to so many rows a block takes all of an expert's, and the second launch is saved (a training pass through 64 experts of 128 -> 128 with 8 rows, whose time is the host's: 30.4 us with both, 26.6 so).
// us of a call in bf16 so, and in tiles with sums: 8 rows of 64 experts, 128 columns 4.3, 7.2; 256 of eight, 1024 5.2, 7.4; 500 of a hundred, 1024 5.4, 12.3; 512 of eight, 4096 7.0, 9.3.  It loses where one or
// a few experts have all rows, which leave few blocks with long turns: 512 of four, 1024 8.8, 7.5; 300 of one, 512 14.8, 7.3; 512 of one, 4096 23.1, 8.7, in fp32 1024 28.7, 8.0.
constexpr int ALL_ROWS = 512;
int wide_tiles(int cols) { return (cols + WIDE - 1) / WIDE; }
int tall_of(long long rows, int cols) { return rows / 128 * wide_tiles(cols) >= 512 ? 128 : 32; }

// A lane has eight columns of every sixteenth row, U of them in flight.  ALL: a block takes all rows of an expert (or those of none), and `partial` is dbias itself.
template <typename T, bool VEC, bool PAST, int U, bool ALL>
__global__ __launch_bounds__(256, 4) void act_back_kernel(ActBackArgs a) {
  __shared__ __align__(16) float part[AT][WIDE + 4];
  const int lane = threadIdx.x % LANES, rows_at = threadIdx.x / LANES, wide = (a.cols + WIDE - 1) / WIDE;
  for (long long at = blockIdx.x; at < a.tiles * wide; at += gridDim.x) {
    const long long tile = at / wide;
    const int col0 = (int)(at - tile * wide) * WIDE, col = col0 + lane * 8, left = a.cols - col;
    int group, row, end;
    if (ALL) {
      group = (int)tile;
      group_rows(a.offs, a.groups, a.rows, group, row, end);
    } else {
      if (!find_tile(a.offs, a.groups, a.rows, a.tall, (unsigned)tile, group, row, end)) return;  // (no later tile either)
      end = min(end, row + a.tall);
    }
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    for (int r0 = row + rows_at; r0 < end; r0 += AT * U) {
      Raw8<T> raw_d[U], raw_z[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = r0 + AT * u, some = r < end ? left : 0;
        raw_d[u].template load<VEC>((const T*)a.dy + r * a.dy_stride + col, some);
        if (a.act != GAN_ACT_NONE) raw_z[u].template load<VEC>((const T*)a.z + r * a.z_stride + col, some);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = r0 + AT * u;
        float d[8], z[8];
        raw_d[u].values(d);
        raw_z[u].values(z);
        times_slope<sizeof(T) == 2 ? FULL : EXACT>(a.act, d, z);                                   // (the bias's gradient is fp32)
        if (group == a.groups)
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] = 0.f;
        if (a.dz) store8<T, VEC, PAST>((T*)a.dz + r * a.dz_stride + col, r < end ? left : 0, d);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += d[i];
      }
    }
    if (!a.partial || (ALL && group == a.groups)) continue;
    __syncthreads();
    *reinterpret_cast<float4*>(&part[rows_at][lane * 8]) = make_float4(sum[0], sum[1], sum[2], sum[3]);
    *reinterpret_cast<float4*>(&part[rows_at][lane * 8 + 4]) = make_float4(sum[4], sum[5], sum[6], sum[7]);
    __syncthreads();
    for (int c = threadIdx.x; c < WIDE; c += 256) {
      float s[AT];
#pragma unroll
      for (int k = 0; k < AT; ++k) s[k] = part[k][c];
#pragma unroll
      for (int k = AT / 2; k > 0; k /= 2)
#pragma unroll
        for (int i = 0; i < k; ++i) s[i] += s[i + k];
      if (col0 + c < a.cols) a.partial[tile * a.cols + col0 + c] = s[0];
    }
  }
}

// dbias: the sums of each expert's tiles.  Eight waves take every eighth tile, in eight chains each, which are joined in order (one expert with most of 15931 rows of 128 columns, 500 tiles of 32
// rows: 5.5 us, by one wave 35).
constexpr int SUM_WAVES = 8;
__global__ __launch_bounds__(64 * SUM_WAVES) void bias_sum_kernel(const int* offs, int groups, int rows, int cols, int tall, const float* partial, float* dbias) {
  __shared__ float part[SUM_WAVES][64];
  const int wide = (cols + 63) / 64, l = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (long long at = blockIdx.x; at < (long long)groups * wide; at += gridDim.x) {
    const int group = (int)(at / wide), col = (int)(at - (long long)group * wide) * 64 + l;
    // the tiles of the experts before
    unsigned first = 0, count = 0;
    int done = 0;
    for (int g0 = 0; g0 <= group; g0 += 64) {
      const int g = g0 + l;
      int hi = g < groups ? min(max(offs[g + 1], 0), rows) : rows;
      hi = max(wave_scan_max(hi), done);
      int lo = __shfl_up(hi, 1);
      if (l == 0) lo = done;
      const unsigned tiles = ((unsigned)(hi - lo) + tall - 1) / tall;
      const unsigned upto = first + (unsigned)wave_scan_add((int)tiles);
      if (group < g0 + 64) {
        count = (unsigned)__shfl((int)tiles, group - g0);
        first = (unsigned)__shfl((int)(upto - tiles), group - g0);
        break;
      }
      done = __shfl(hi, 63);
      first = (unsigned)__shfl((int)upto, 63);
    }
    float s[8] = {};
    if (col < cols)
      for (unsigned t = wave; t < count; t += 8 * SUM_WAVES) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = t + SUM_WAVES * k < count ? partial[(long long)(first + t + SUM_WAVES * k) * cols + col] : 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += v[k];
      }
    __syncthreads();                                              // (the last turn's have been read)
    part[wave][l] = ((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]));
    __syncthreads();
    if (wave == 0 && col < cols) {
      float d = part[0][l];
#pragma unroll
      for (int w = 1; w < SUM_WAVES; ++w) d += part[w][l];
      dbias[(long long)group * cols + col] = d;
    }
  }
}

}  // namespace
}  // namespace gan

using namespace gan;

extern "C" int64_t gan_group_act_backward_bytes(int32_t groups, int64_t rows, int32_t cols) {
  if (groups < 1 || rows <= ALL_ROWS || cols < 1 || groups > 65535 || rows > MOST_ROWS || cols > MOST_COLS) return 0;
  return most_tiles(rows, groups, tall_of(rows, cols)) * cols * (int64_t)sizeof(float);
}

extern "C" gan_status gan_group_act_backward(int32_t precision, const void* dy, int64_t dy_stride, int32_t act, const void* z, int64_t z_stride, const int32_t* offs,
                                             int32_t groups, int64_t rows, int32_t cols, void* dz, int64_t dz_stride, float* dbias, void* work, int64_t work_bytes,
                                             void* hip_stream) {
  if (const gan_status s = check_sizes(precision, rows, cols)) return s;
  if (!act_known(act)) return operator_fail(GAN_E_ARG, "unknown activation");
  if (groups < 0) return operator_fail(GAN_E_ARG, "negative groups");
  if (groups > 65535) return operator_fail(GAN_E_SHAPE, "more than 65535 groups");
  if (!offs || (rows > 0 && (!dy || (act != GAN_ACT_NONE && !z)))) return operator_fail(GAN_E_ARG, "dy, z or offs is NULL");
  for (const gan_status s : {check_matrix(dy, dy_stride, cols, "dy_stride is below cols"), check_matrix(act != GAN_ACT_NONE ? z : nullptr, z_stride, cols, "z_stride is below cols"),
                             check_matrix(dz, dz_stride, cols, "dz_stride is below cols")})
    if (s) return s;
  const int64_t need = gan_group_act_backward_bytes(groups, rows, cols);
  if (dbias && (work_bytes < need || (need > 0 && !work) || !aligned16(work)))
    return operator_fail(GAN_E_ARG, "work is smaller than gan_group_act_backward_bytes, or not 16-byte aligned");
  if (!dbias && !dz) return GAN_OK;
  operator_launches();
  const hipStream_t st = (hipStream_t)hip_stream;
  const int e = precision == GAN_FP32 ? 4 : 2;
  if (rows > 0) {
    const bool vec = cols % 8 == 0 && rows_aligned16(dy, dy_stride, e) && (act == GAN_ACT_NONE || rows_aligned16(z, z_stride, e)) && (!dz || rows_aligned16(dz, dz_stride, e));
    const int tall = tall_of(rows, cols);
    const bool all = rows <= ALL_ROWS, past = rows * cols * e > PAST_CACHES;
    float* const partial = dbias && groups > 0 ? all ? dbias : (float*)work : nullptr;
    const ActBackArgs a = {dy, z, offs, dz, partial, dy_stride, z_stride, dz_stride, groups, (int)rows, cols, act, tall, all ? groups + 1 : most_tiles(rows, groups, tall)};
    const dim3 grid((unsigned)std::min(a.tiles * wide_tiles(cols), 1ll << 20));
#define GAN_ACT_BACK(T, V) \
  if (all) hipLaunchKernelGGL((act_back_kernel<T, V, false, 2, true>), grid, dim3(256), 0, st, a); \
  else if (tall == 32) hipLaunchKernelGGL((act_back_kernel<T, V, false, 2, false>), grid, dim3(256), 0, st, a); \
  else if (V && past) hipLaunchKernelGGL((act_back_kernel<T, V, V, 4, false>), grid, dim3(256), 0, st, a); \
  else hipLaunchKernelGGL((act_back_kernel<T, V, false, 4, false>), grid, dim3(256), 0, st, a)
    if (precision == GAN_FP32) { if (vec) { GAN_ACT_BACK(float, true); } else { GAN_ACT_BACK(float, false); } }
    else { if (vec) { GAN_ACT_BACK(bf16_t, true); } else { GAN_ACT_BACK(bf16_t, false); } }
#undef GAN_ACT_BACK
  }
  if (dbias && groups > 0 && (rows == 0 || rows > ALL_ROWS)) {
    const long long blocks = groups * (((long long)cols + 63) / 64);
    hipLaunchKernelGGL(bias_sum_kernel, dim3((unsigned)std::min(blocks, 1ll << 20)), dim3(64 * SUM_WAVES), 0, st, offs, groups, (int)rows, cols, tall_of(rows, cols), (const float*)work, dbias);
  }
  return operator_launched();
}

// The gradient through the activation behind a product grouped by label, with the bias's gradient on the way.
//
//   dz = dy act'(z),    dbias[g] = sum of dz over g's rows
//
// Bound by memory, one pass over dy and z.  Blocks take tiles of rows of one expert each and some columns, and leave the sums of their rows, which a second kernel adds up expert
// by expert, in order.
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
  long long tiles;                                                // of rows, at most
};

constexpr int TALL = 64;                                          // rows of a tile

// Four waves of 64 lanes, eight columns each: wave w takes the rows w, w + 4, ...
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void act_back_kernel(ActBackArgs a) {
  __shared__ float part[4][512];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wide = (a.cols + 511) / 512;
  for (long long at = blockIdx.x; at < a.tiles * wide; at += gridDim.x) {
    const long long tile = at / wide;
    const int col = ((int)(at - tile * wide) * 64 + lane) * 8, left = a.cols - col;
    int group, row, end;
    if (!find_tile(a.offs, a.groups, a.rows, TALL, (unsigned)tile, group, row, end)) return;      // (no later tile either)
    end = min(end, row + TALL);
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    for (int r = row + wave; r < end; r += 4) {
      float d[8], z[8];
      load8<T, VEC>((const T*)a.dy + r * a.dy_stride + col, left, d);
      if (a.act != GAN_ACT_NONE) {
        load8<T, VEC>((const T*)a.z + r * a.z_stride + col, left, z);
        times_slope<false>(a.act, d, z);                          // (the bias's gradient is fp32)
      }
      if (group == a.groups)
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = 0.f;
      if (a.dz) store8<T, VEC>((T*)a.dz + r * a.dz_stride + col, left, d);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += d[i];
    }
    if (!a.partial) continue;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) part[wave][lane * 8 + i] = sum[i];
    __syncthreads();
    for (int c = threadIdx.x; c < 512; c += 256) {
      const int to = (int)(at - tile * wide) * 512 + c;
      if (to < a.cols) a.partial[tile * a.cols + to] = (part[0][c] + part[1][c]) + (part[2][c] + part[3][c]);
    }
  }
}

// dbias: the sums of each expert's tiles, in order
__global__ __launch_bounds__(256) void bias_sum_kernel(const int* offs, int groups, int rows, int cols, const float* partial, float* dbias) {
  const int wide = (cols + 255) / 256;
  for (long long at = blockIdx.x; at < (long long)groups * wide; at += gridDim.x) {
    const int group = (int)(at / wide), col = (int)(at - (long long)group * wide) * 256 + threadIdx.x;
    // the tiles of the experts before
    unsigned first = 0, count = 0;
    int done = 0;
    const int l = threadIdx.x & 63;
    for (int g0 = 0; g0 <= group; g0 += 64) {
      const int g = g0 + l;
      int hi = g < groups ? min(max(offs[g + 1], 0), rows) : rows;
      hi = max(wave_scan_max(hi), done);
      int lo = __shfl_up(hi, 1);
      if (l == 0) lo = done;
      const unsigned tiles = ((unsigned)(hi - lo) + TALL - 1) / TALL;
      const unsigned upto = first + (unsigned)wave_scan_add((int)tiles);
      if (group < g0 + 64) {
        count = (unsigned)__shfl((int)tiles, group - g0);
        first = (unsigned)__shfl((int)(upto - tiles), group - g0);
        break;
      }
      done = __shfl(hi, 63);
      first = (unsigned)__shfl((int)upto, 63);
    }
    if (col >= cols) continue;
    float s = 0.f;
    for (unsigned t = 0; t < count; ++t) s += partial[(long long)(first + t) * cols + col];
    dbias[(long long)group * cols + col] = s;
  }
}

}  // namespace
}  // namespace gan

using namespace gan;

extern "C" int64_t gan_group_act_backward_bytes(int32_t groups, int64_t rows, int32_t cols) {
  if (groups < 1 || rows < 1 || cols < 1 || groups > 65535 || rows > MOST_ROWS || cols > MOST_COLS) return 0;
  return most_tiles(rows, groups, TALL) * cols * (int64_t)sizeof(float);
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
    const ActBackArgs a = {dy, z, offs, dz, dbias && groups > 0 ? (float*)work : nullptr, dy_stride, z_stride, dz_stride, groups, (int)rows, cols, act,
                           most_tiles(rows, groups, TALL)};
    const dim3 grid((unsigned)std::min(a.tiles * ((cols + 511) / 512), 1ll << 20));
#define GAN_ACT_BACK(T, V) hipLaunchKernelGGL((act_back_kernel<T, V>), grid, dim3(256), 0, st, a)
    if (precision == GAN_FP32) { if (vec) GAN_ACT_BACK(float, true); else GAN_ACT_BACK(float, false); }
    else { if (vec) GAN_ACT_BACK(bf16_t, true); else GAN_ACT_BACK(bf16_t, false); }
#undef GAN_ACT_BACK
  }
  if (dbias && groups > 0) {
    const long long blocks = groups * (((long long)cols + 255) / 256);
    hipLaunchKernelGGL(bias_sum_kernel, dim3((unsigned)std::min(blocks, 1ll << 20)), dim3(256), 0, st, offs, groups, (int)rows, cols, (const float*)work, dbias);
  }
  return operator_launched();
}

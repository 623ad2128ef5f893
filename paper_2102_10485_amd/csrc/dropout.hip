// Dropout with the residual's addition; its gradient is the same call.
//
//   y = residual + keep * x / (1 - p)
//
// Whether an element is kept follows from its place alone: Philox-4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC'11) gives 128 bits
// for every eight neighbours of a row, sixteen for each of them, so that no mask is stored and no state kept.  Bound by memory, two or three passes: bf16 on an MI355X, 16384 x 4096 with a
// residual 63 us (6.4 TB/s) and without one 47 (5.7); the generator's twenty 64-bit products for eight elements stay below that.  Results of more than 64 MiB go past the caches (through them
// 72 and 52).  Two chunks a thread are in flight (one: 66 and 49; four: 66 and 48, and 1117 x 1000 in fp32 4.6 for 4.0).
#include "row_chunks.h"

namespace gan {
namespace {

struct DropoutArgs {
  const void *x, *residual;
  void* y;
  const uint32_t* step_device;
  long long x_stride, residual_stride, y_stride;
  RowChunks s;
  int cols;
  unsigned threshold;                                             // of 65536: fewer are dropped
  float scale;
  unsigned seed_lo, seed_hi, site, step;
};

// A round maps (c0, c1, c2, c3) to (hi(M1 c2) ^ c1 ^ k0, lo(M1 c2), hi(M0 c0) ^ c3 ^ k1, lo(M0 c0)); two Weyl constants advance the key between rounds.
__device__ __forceinline__ void philox(unsigned (&c)[4], unsigned k0, unsigned k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long a = (unsigned long long)0xD2511F53u * c[0], b = (unsigned long long)0xCD9E8D57u * c[2];
    c[0] = (unsigned)(b >> 32) ^ c[1] ^ k0;
    c[2] = (unsigned)(a >> 32) ^ c[3] ^ k1;
    c[1] = (unsigned)b;
    c[3] = (unsigned)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

constexpr int DROP_EACH = 2, DROP_TILE = 256 * DROP_EACH;         // chunks of a thread, and of a block, a turn

template <typename T, bool VEC, bool PAST>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a) {
  const unsigned step = a.step + (a.step_device ? *a.step_device : 0u);
  const long long chunks = a.s.rows * a.s.eights;
  for (long long first = (long long)blockIdx.x * DROP_TILE; first < chunks; first += (long long)gridDim.x * DROP_TILE) {
    const long long row0 = first / a.s.eights;
    const unsigned col0 = (unsigned)(first - row0 * a.s.eights);
    Raw8<T> x[DROP_EACH], res[DROP_EACH];
    long long row[DROP_EACH];
    int col[DROP_EACH], left[DROP_EACH];
#pragma unroll
    for (int u = 0; u < DROP_EACH; ++u) {
      const unsigned t = u * 256 + threadIdx.x;
      unsigned chunk;
      chunk_at(a.s, row0, col0, t, row[u], chunk);
      col[u] = (int)chunk * 8;
      left[u] = first + t < chunks ? a.cols - col[u] : 0;
      x[u].template load<VEC>((const T*)a.x + row[u] * a.x_stride + col[u], left[u]);
      if (a.residual) res[u].template load<VEC>((const T*)a.residual + row[u] * a.residual_stride + col[u], left[u]);
    }
#pragma unroll
    for (int u = 0; u < DROP_EACH; ++u) {
      const unsigned long long q = (unsigned long long)(first + u * 256 + threadIdx.x);
      unsigned c[4] = {(unsigned)q, (unsigned)(q >> 32), a.site, step};
      philox(c, a.seed_lo, a.seed_hi);
      float v[8], r[8];
      x[u].values(v);
      if (a.residual) res[u].values(r);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const unsigned bits = i % 2 ? c[i / 2] >> 16 : c[i / 2] & 0xffffu;
        v[i] = bits >= a.threshold ? v[i] * a.scale : 0.f;
        if (a.residual) v[i] += r[i];
      }
      store8<T, VEC, PAST>((T*)a.y + row[u] * a.y_stride + col[u], left[u], v);
    }
  }
}

}  // namespace
}  // namespace gan

using namespace gan;

extern "C" gan_status gan_dropout(int32_t precision, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, int64_t rows, int32_t cols, double p,
                                  uint64_t seed, uint32_t site, uint32_t step, const uint32_t* step_device, void* y, int64_t y_stride, void* hip_stream) {
  if (const gan_status s = check_sizes(precision, rows, cols)) return s;
  if (rows > 0 && (!x || !y)) return operator_fail(GAN_E_ARG, "x or y is NULL");
  if (!(p >= 0 && p < 1)) return operator_fail(GAN_E_ARG, "p is outside [0, 1)");
  for (const gan_status s : {check_matrix(x, x_stride, cols, "x_stride is below cols"), check_matrix(residual, residual_stride, cols, "residual_stride is below cols"),
                             check_matrix(y, y_stride, cols, "y_stride is below cols")})
    if (s) return s;
  const unsigned threshold = (unsigned)(p * 65536 + 0.5);
  if (threshold == 65536) return operator_fail(GAN_E_ARG, "p is 1 in steps of 2^-16");
  if (rows == 0) return GAN_OK;
  operator_launches();
  const int e = precision == GAN_FP32 ? 4 : 2;
  const bool vec = cols % 8 == 0 && rows_aligned16(x, x_stride, e) && (!residual || rows_aligned16(residual, residual_stride, e)) && rows_aligned16(y, y_stride, e);
  const DropoutArgs a = {x, residual, y, step_device, x_stride, residual_stride, y_stride, row_chunks(rows, cols), cols, threshold, 65536.f / (float)(65536 - threshold),
                         (unsigned)seed, (unsigned)(seed >> 32), site, step};
  const dim3 grid(chunk_blocks(a.s, DROP_TILE, 1 << 20));
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool past = rows * cols * e > PAST_CACHES;
#define GAN_DROPOUT(T, V) \
  if (V && past) hipLaunchKernelGGL((dropout_kernel<T, V, V>), grid, dim3(256), 0, st, a); \
  else hipLaunchKernelGGL((dropout_kernel<T, V, false>), grid, dim3(256), 0, st, a)
  if (precision == GAN_FP32) { if (vec) { GAN_DROPOUT(float, true); } else { GAN_DROPOUT(float, false); } }
  else { if (vec) { GAN_DROPOUT(bf16_t, true); } else { GAN_DROPOUT(bf16_t, false); } }
#undef GAN_DROPOUT
  return operator_launched();
}

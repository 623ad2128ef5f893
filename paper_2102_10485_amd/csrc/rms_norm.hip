// The root-mean-square norm of rows with the residual's addition, its gradient, and matrices into 8 bits.
//
//   sum = round(x + residual), inv = 1 / sqrt(mean(sum^2) + eps), y = sum * inv * gain
//
// Bound by memory: one pass over x and residual, six operations an element; bf16 on an MI355X: 16384 x 4096 into 8 bits 81-84 us (5.6-5.8 TB/s), 6400 x 2048 forward 21 us and
// gradient 25 us from cold memory (5.1 and 4.1 TB/s; a plain copy 4.9), four rows of 1024 3.2 us.  A row is held in registers between the sum of its squares and
// its output, by one wave (up to 512 elements, 1024 in many rows, where no barrier is needed), a block of four waves, or one of sixteen; rows beyond
// 32768 elements (16384 in the gradient) are read a second time.
#include "operators.h"

namespace gan {
namespace {

constexpr int E = 8;                                              // elements of a lane's chunk

template <int WAVES>
__device__ __forceinline__ float row_total(float v, float* scratch) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  if constexpr (WAVES > 1) {
    __syncthreads();                                              // (what the last row left in scratch has been read)
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += scratch[w];
  }
  return v;
}

struct NormArgs {
  const void *x, *residual;
  const float* gain;
  void *sum, *y;
  uint8_t *y8, *y8_scale;
  float* inv_rms;
  long long x_stride, residual_stride, sum_stride, y_stride, rows;
  int cols;
  float eps;
};

// Results of more bytes than this go past the caches, which would not hold them all for their reader (bf16 with the sum, us through the caches and past them:
// 16384 x 4096 94.6, 76.2, into 8 bits 86.7, 70.3; 65536 x 512 48.5, 39.5; 12000 x 2048 37.5, 34.3; a norm and two products of four experts on 16384 x 4096
// 950, 942; the gradient of 40000 x 1024 58.7, 50.5, of 16384 x 4096 98, 96).  Smaller ones stay for it (norm and products of eight experts of 128 rows of 1024: 34.4, past the caches 36.9).
constexpr long long PAST_CACHES = 64 << 20;

template <typename T, bool VEC>
__device__ __forceinline__ void add_rounded(float (&v)[E], const T* residual, int left) {
  float r[E];
  load8<T, VEC>(residual, left, r);
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = to_float(from_float<T>(v[i] + r[i]));
}

template <typename T, bool VEC, bool PAST>
__device__ __forceinline__ void write_chunk(const NormArgs& a, long long row, int col, const float (&s)[E], float inv) {
  float g[E], y[E];
  const int left = a.cols - col;
  load8<float, VEC>(a.gain + col, left, g);
#pragma unroll
  for (int i = 0; i < E; ++i) y[i] = (VEC ? left > 0 : i < left) ? s[i] * inv * g[i] : 0.f;       // (behind the row inv may be NaN or infinite, and the codes are zero)
  if (a.y) store8<T, VEC, PAST>((T*)a.y + row * a.y_stride + col, left, y);
  if (a.y8) {                                                     // the sixteen lanes of a block of 128 are here together, or none is
    const long long padded = padded8(a.cols);
    const int byte = scale_byte(y);
    store_codes<PAST>(a.y8 + row * padded + col, to_e4m3_x8(y, byte));
    if ((threadIdx.x & 15) == 0) a.y8_scale[(row * padded + col) / BLOCK8] = (uint8_t)byte;
  }
}

// WAVES waves a row, lane l of them holding the chunks l, l + 64 WAVES, ...; blocks of four rows where a row is a wave's
template <typename T, int WAVES, int CHUNKS, bool VEC, bool PAST>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void norm_kernel(NormArgs a) {
  __shared__ float scratch[WAVES];
  const long long row = WAVES == 1 ? (long long)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (row >= a.rows) return;                                      // (whole waves; blocks of several waves have one row)
  const int lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  float s[CHUNKS][E];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int col = (c * 64 * WAVES + lane) * E;
    load8<T, VEC>((const T*)a.x + row * a.x_stride + col, a.cols - col, s[c]);
  }
  if (a.residual)
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int col = (c * 64 * WAVES + lane) * E;
      add_rounded<T, VEC>(s[c], (const T*)a.residual + row * a.residual_stride + col, a.cols - col);
    }
  float q = 0.f;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int col = (c * 64 * WAVES + lane) * E;
    if (a.sum) store8<T, VEC, PAST>((T*)a.sum + row * a.sum_stride + col, a.cols - col, s[c]);
#pragma unroll
    for (int i = 0; i < E; ++i) q += s[c][i] * s[c][i];
  }
  const float inv = 1.f / sqrtf(row_total<WAVES>(q, scratch) / (float)a.cols + a.eps);
  if (a.inv_rms && lane == 0) a.inv_rms[row] = inv;
  if (!a.y && !a.y8) return;
  const int wide = (int)padded8(a.cols);
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int col = (c * 64 * WAVES + lane) * E;
    if (col < wide) write_chunk<T, VEC, PAST>(a, row, col, s[c], inv);
  }
}

// Rows of any length: the sum is formed again for the output (from `sum`, where it was stored over an operand).
template <typename T, bool VEC>
__global__ __launch_bounds__(1024) void norm_long_kernel(NormArgs a) {
  __shared__ float scratch[16];
  const long long row = blockIdx.x;
  const T* x = (const T*)a.x + row * a.x_stride;
  const T* residual = a.residual ? (const T*)a.residual + row * a.residual_stride : nullptr;
  T* sum = a.sum ? (T*)a.sum + row * a.sum_stride : nullptr;
  float q = 0.f, s[E];
  for (int col = threadIdx.x * E; col < a.cols; col += 1024 * E) {
    load8<T, VEC>(x + col, a.cols - col, s);
    if (residual) add_rounded<T, VEC>(s, residual + col, a.cols - col);
    if (sum) store8<T, VEC>(sum + col, a.cols - col, s);
#pragma unroll
    for (int i = 0; i < E; ++i) q += s[i] * s[i];
  }
  const float inv = 1.f / sqrtf(row_total<16>(q, scratch) / (float)a.cols + a.eps);
  if (a.inv_rms && threadIdx.x == 0) a.inv_rms[row] = inv;
  if (!a.y && !a.y8) return;
  const int wide = (int)padded8(a.cols);
  for (int col = threadIdx.x * E; col < wide; col += 1024 * E) {
    if (sum) {
      load8<T, VEC>(sum + col, a.cols - col, s);                  // (this thread's own stores)
    } else {
      load8<T, VEC>(x + col, a.cols - col, s);
      if (residual) add_rounded<T, VEC>(s, residual + col, a.cols - col);
    }
    write_chunk<T, VEC, false>(a, row, col, s, inv);
  }
}

// A launch has fewer than 2^32 threads (the runtime takes more of them modulo 2^32, without an error): `go` is called with the first of `count` shares of `waves` waves each,
// and with how many of them a launch takes.
template <typename F>
void by_launches(long long count, int waves, F&& go) {
  const long long most = (1ll << 31) / (64 * waves);
  for (long long first = 0; first < count; first += most) go(first, count - first < most ? count - first : most);
}

template <typename T>
NormArgs rows_of(NormArgs a, long long first, long long rows) {
  const long long wide = padded8(a.cols);
  a.x = (const T*)a.x + first * a.x_stride;
  if (a.residual) a.residual = (const T*)a.residual + first * a.residual_stride;
  if (a.sum) a.sum = (T*)a.sum + first * a.sum_stride;
  if (a.y) a.y = (T*)a.y + first * a.y_stride;
  if (a.y8) a.y8 += first * wide, a.y8_scale += first * (wide / BLOCK8);
  if (a.inv_rms) a.inv_rms += first;
  a.rows = rows;
  return a;
}

template <typename T, int WAVES, int CHUNKS, bool VEC, bool PAST>
void launch_norm_as(const NormArgs& a, hipStream_t st) {
  by_launches(a.rows, WAVES, [&](long long first, long long rows) {
    hipLaunchKernelGGL((norm_kernel<T, WAVES, CHUNKS, VEC, PAST>), dim3((unsigned)(WAVES == 1 ? (rows + 3) / 4 : rows)), dim3(WAVES == 1 ? 256 : 64 * WAVES), 0, st,
                       rows_of<T>(a, first, rows));
  });
}

template <typename T, bool VEC, bool PAST>
void launch_norm(const NormArgs& a, hipStream_t st) {
  const long long cols = a.cols;
#define GAN_NORM(W, C) launch_norm_as<T, W, C, VEC, PAST>(a, st)
  // Times on an MI355X.  Up to 1024 elements a wave per row has no barrier (bf16, 6400 x 1024: 13.5 us, four waves a row 15.6), but few rows
  // are done sooner by more waves (fp32, 1117 x 1000: 6.4 and 6.0).  Above, one chunk a lane is faster than more of them in fewer waves (bf16, 6400 x 2048: 22.8 us by four
  // waves, 28.7 by one; 4096 x 8192: 48.6 by sixteen, 52.9 by four).
  if (cols <= 512) GAN_NORM(1, 1);
  else if (cols <= 1024 && a.rows >= 4096) GAN_NORM(1, 2);
  else if (cols <= 2048) GAN_NORM(4, 1);
  else if (cols <= 4096) GAN_NORM(4, 2);
  else if (cols <= 8192) GAN_NORM(16, 1);
  else if (cols <= 16384) GAN_NORM(16, 2);
  else if (cols <= 32768) GAN_NORM(16, 4);
  else
    by_launches(a.rows, 16, [&](long long first, long long rows) {
      hipLaunchKernelGGL((norm_long_kernel<T, VEC>), dim3((unsigned)rows), dim3(1024), 0, st, rows_of<T>(a, first, rows));
    });
#undef GAN_NORM
}

// ---- gradient ----

struct NormBackArgs {
  const void *dy, *sum, *dsum;
  const float *gain, *inv_rms;
  void* dx;
  float* partial;                                                 // [blocks][cols]: the gain's gradient of each block's rows, or NULL
  long long dy_stride, sum_stride, dsum_stride, dx_stride, rows;
  int cols;
};

// What a lane holds of a row as it is stored: eight elements.
template <typename T> struct Raw { uint4 v[sizeof(T) / 2]; };
template <typename T, bool VEC>
__device__ __forceinline__ Raw<T> load_raw(const T* p, int left) {
  Raw<T> r;
  if (left >= 8) {
    typedef typename Words<VEC ? 16 : sizeof(T)>::T words;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = __builtin_bit_cast(uint4, reinterpret_cast<const words*>(p)[i]);
  } else {
    T e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = !VEC && i < left ? p[i] : from_float<T>(0.f);
    __builtin_memcpy(&r, e, sizeof(r));
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void unpack(const Raw<T>& r, float (&v)[E]) {
  T e[8];
  __builtin_memcpy(e, &r, sizeof(r));
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = to_float(e[i]);
}

// A row's share of the gain's gradient stays in its lanes' registers over all rows of the wave, and the next row is loaded while this one is worked on (both launches of 6400 x 2048 in bf16: 47.9 -> 28.8 us); four
// waves of one row each are joined at the end.
template <typename T, int WAVES, int CHUNKS, bool VEC, bool PAST>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) void norm_back_kernel(NormBackArgs a) {
  __shared__ float scratch[WAVES == 1 ? 4 * 64 * E : WAVES];
  const int lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  const int wave = WAVES == 1 ? threadIdx.x >> 6 : 0;
  const long long step = (long long)gridDim.x * (WAVES == 1 ? 4 : 1);
  float dg[CHUNKS][E];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int i = 0; i < E; ++i) dg[c][i] = 0.f;
  struct Row { Raw<T> dy[CHUNKS], s[CHUNKS], ds[CHUNKS]; float inv; } next;
  auto load_row = [&](long long row) {
    next.inv = a.inv_rms[row];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int col = (c * 64 * WAVES + lane) * E, left = a.cols - col;
      next.dy[c] = load_raw<T, VEC>((const T*)a.dy + row * a.dy_stride + col, left);
      next.s[c] = load_raw<T, VEC>((const T*)a.sum + row * a.sum_stride + col, left);
      next.ds[c] = load_raw<T, VEC>((const T*)a.dsum + row * a.dsum_stride + col, a.dsum ? left : 0);
    }
  };
  long long row = WAVES == 1 ? (long long)blockIdx.x * 4 + wave : blockIdx.x;
  if (row < a.rows) load_row(row);
  for (; row < a.rows; row += step) {
    if (WAVES == 16 && row >= gridDim.x) load_row(row);           // (no registers for two rows)
    const Row now = next;
    if (WAVES < 16 && row + step < a.rows) load_row(row + step);
    float s[CHUNKS][E], h[CHUNKS][E], dot = 0.f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int col = (c * 64 * WAVES + lane) * E;
      float g[E];
      load8<float, VEC>(a.gain + col, a.cols - col, g);
      unpack<T>(now.dy[c], h[c]);
      unpack<T>(now.s[c], s[c]);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        dg[c][i] += h[c][i] * (s[c][i] * now.inv);
        h[c][i] *= g[i];
        dot += h[c][i] * s[c][i];
      }
    }
    const float k = now.inv * (now.inv * (row_total<WAVES>(dot, scratch) / (float)a.cols));     // (inv^2 alone may be no fp32 number: rows of 1e-20 without eps)
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int col = (c * 64 * WAVES + lane) * E;
      float d[E];
      unpack<T>(now.ds[c], d);
#pragma unroll
      for (int i = 0; i < E; ++i) d[i] += now.inv * (h[c][i] - s[c][i] * k);
      store8<T, VEC, PAST>((T*)a.dx + row * a.dx_stride + col, a.cols - col, d);
    }
  }
  if (!a.partial) return;
  float* out = a.partial + (long long)blockIdx.x * a.cols;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int col = (c * 64 * WAVES + lane) * E;
    if constexpr (WAVES == 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < E; ++i) scratch[(wave * E + i) * 64 + lane] = dg[c][i];
      __syncthreads();
      if (wave == 0) {
#pragma unroll
        for (int i = 0; i < E; ++i) dg[c][i] = scratch[i * 64 + lane] + scratch[(E + i) * 64 + lane] + scratch[(2 * E + i) * 64 + lane] + scratch[(3 * E + i) * 64 + lane];
        store8<float, false>(out + col, a.cols - col, dg[c]);
      }
    } else {
      store8<float, false>(out + col, a.cols - col, dg[c]);
    }
  }
}

// Rows of any length: the products are formed twice, and the gain's gradient by threads that own columns.
template <typename T, bool VEC>
__global__ __launch_bounds__(1024) void norm_back_long_kernel(NormBackArgs a) {
  __shared__ float scratch[16];
  const long long row = blockIdx.x;
  const T *dy = (const T*)a.dy + row * a.dy_stride, *sum = (const T*)a.sum + row * a.sum_stride;
  const float inv = a.inv_rms[row];
  float h[E], s[E], g[E], dot = 0.f;
  for (int col = threadIdx.x * E; col < a.cols; col += 1024 * E) {
    load8<T, VEC>(dy + col, a.cols - col, h);
    load8<T, VEC>(sum + col, a.cols - col, s);
    load8<float, VEC>(a.gain + col, a.cols - col, g);
#pragma unroll
    for (int i = 0; i < E; ++i) dot += h[i] * g[i] * s[i];
  }
  const float k = inv * (inv * (row_total<16>(dot, scratch) / (float)a.cols));
  for (int col = threadIdx.x * E; col < a.cols; col += 1024 * E) {
    load8<T, VEC>(dy + col, a.cols - col, h);
    load8<T, VEC>(sum + col, a.cols - col, s);
    load8<float, VEC>(a.gain + col, a.cols - col, g);
    float d[E];
    if (a.dsum) {
      load8<T, VEC>((const T*)a.dsum + row * a.dsum_stride + col, a.cols - col, d);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) d[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < E; ++i) d[i] += inv * (h[i] * g[i] - s[i] * k);
    store8<T, VEC>((T*)a.dx + row * a.dx_stride + col, a.cols - col, d);
  }
}
template <typename T>
__global__ __launch_bounds__(256) void gain_long_kernel(NormBackArgs a) {
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= a.cols) return;
  float d = 0.f;
  for (long long row = blockIdx.y; row < a.rows; row += gridDim.y)
    d += to_float(((const T*)a.dy)[row * a.dy_stride + col]) * (to_float(((const T*)a.sum)[row * a.sum_stride + col]) * a.inv_rms[row]);
  a.partial[(long long)blockIdx.y * a.cols + col] = d;
}

// dgain[c] = the blocks' partial sums, added in 32 chains that are joined in order; eight loads of a chain in flight
__global__ __launch_bounds__(1024) void gain_sum_kernel(const float* partial, float* dgain, int blocks, int cols, int first_col) {
  __shared__ float part[32][33];
  const int c = threadIdx.x & 31, k = threadIdx.x >> 5, col = first_col + blockIdx.x * 32 + c;
  float d = 0.f;
  if (col < cols)
    for (int b = k; b < blocks; b += 256) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = b + 32 * i < blocks ? partial[(long long)(b + 32 * i) * cols + col] : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) d += v[i];
    }
  part[k][c] = d;
  __syncthreads();
  if (k == 0 && col < cols) {
#pragma unroll
    for (int j = 1; j < 32; ++j) d += part[j][c];
    dgain[col] = d;
  }
}

constexpr int REGISTER_COLS = 16384;                              // rows that norm_back_kernel holds

// Blocks of the gradient: each leaves a row of partial sums, which twice as many would make slower to add than they gain (bf16, 16384 x 4096: 98 us with 512
// blocks, 109 with 1024).
int back_blocks(long long rows, int cols) {
  if (cols > REGISTER_COLS) return (int)(rows < 64 ? rows : 64);
  const long long per = cols <= 1024 ? 4 : 1, blocks = (rows + per - 1) / per, most = cols > 1024 && cols <= 2048 ? 1024 : cols <= 8192 ? 512 : 256;
  return (int)(blocks < most ? blocks : most);
}

template <typename T, bool VEC, bool PAST>
void launch_back(const NormBackArgs& a, hipStream_t st) {
  const unsigned blocks = (unsigned)back_blocks(a.rows, a.cols);
#define GAN_BACK(W, C) hipLaunchKernelGGL((norm_back_kernel<T, W, C, VEC, PAST>), dim3(blocks), dim3(W == 1 ? 256 : 64 * W), 0, st, a)
  // (bf16, 6400 x 1024: 17.1 us with a wave a row, 20.1 with four; fp32, 4000 x 2048: 32.8 us with four, 36.7 with one)
  if (a.cols <= 512) GAN_BACK(1, 1);
  else if (a.cols <= 1024) GAN_BACK(1, 2);
  else if (a.cols <= 2048) GAN_BACK(4, 1);
  else if (a.cols <= 4096) GAN_BACK(4, 2);
  else if (a.cols <= 8192) GAN_BACK(4, 4);
  else if (a.cols <= REGISTER_COLS) GAN_BACK(16, 2);
  else {
    // (the gain's gradient first: dx may be the memory of dy)
    if (a.partial) hipLaunchKernelGGL(gain_long_kernel<T>, dim3((a.cols + 255) / 256, blocks), dim3(256), 0, st, a);
    by_launches(a.rows, 16, [&](long long first, long long rows) {
      NormBackArgs some = a;
      some.dy = (const T*)a.dy + first * a.dy_stride;
      some.sum = (const T*)a.sum + first * a.sum_stride;
      if (a.dsum) some.dsum = (const T*)a.dsum + first * a.dsum_stride;
      some.dx = (T*)a.dx + first * a.dx_stride;
      some.inv_rms += first;
      some.rows = rows;
      hipLaunchKernelGGL((norm_back_long_kernel<T, VEC>), dim3((unsigned)rows), dim3(1024), 0, st, some);
    });
  }
#undef GAN_BACK
}

// ---- 8 bits ----
//
// Bound by memory, a pass that reads a matrix and writes half or a quarter of its bytes: bf16, 16384 x 4096 44 us (4.6 TB/s), 32768 x 4096 74 (5.4), 6400 x 2048 9.3, fp32, 40960 x 4096 165 (5.1); up to a
// million values the launch (3.8).  Sixteen lanes hold a block of 128, so that its scale is four exchanges between lanes.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void quantize8_kernel(const T* x, long long stride, long long rows, int cols, uint8_t* q, uint8_t* scale) {
  const long long wide = padded8(cols), chunks = rows * (wide / E);
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (long long)gridDim.x * 256) {   // (sixteen lanes of a block stay together)
    const long long row = i * E / wide;
    const int col = (int)(i * E - row * wide);
    float v[E];
    load8<T, VEC>(x + row * stride + col, cols - col, v);
    const int byte = scale_byte(v);
    *reinterpret_cast<uint2*>(q + i * E) = to_e4m3_x8(v, byte);
    if ((threadIdx.x & 15) == 0) scale[i * E / BLOCK8] = (uint8_t)byte;
  }
}

constexpr long long MOST_ROWS = 1 << 30;
constexpr int MOST_COLS = 1 << 28;

bool precision_known(int32_t p) { return p == GAN_FP32 || p == GAN_BF16_FP32MASTER; }
gan_status check_matrix(const void* p, long long stride, int cols, const char* why) {
  return p && stride < cols ? operator_fail(GAN_E_ARG, why) : GAN_OK;
}
gan_status check_sizes(int32_t precision, long long rows, int cols) {
  if (!precision_known(precision)) return operator_fail(GAN_E_ARG, "unknown precision");
  if (rows < 0 || cols < 1) return operator_fail(GAN_E_ARG, "negative rows or no columns");
  if (rows > MOST_ROWS || cols > MOST_COLS) return operator_fail(GAN_E_SHAPE, "more than 2^30 rows or 2^28 columns");
  return GAN_OK;
}

}  // namespace
}  // namespace gan

using namespace gan;

extern "C" gan_status gan_rms_norm(int32_t precision, const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const float* gain,
                                   float eps, int64_t rows, int32_t cols, void* sum, int64_t sum_stride, void* y, int64_t y_stride, uint8_t* y8,
                                   uint8_t* y8_scale, float* inv_rms, void* hip_stream) {
  if (const gan_status s = check_sizes(precision, rows, cols)) return s;
  if ((rows > 0 && !x) || !gain) return operator_fail(GAN_E_ARG, "x or gain is NULL");
  if (!y8 != !y8_scale) return operator_fail(GAN_E_ARG, "y8 and y8_scale go together");
  if (!aligned16(y8)) return operator_fail(GAN_E_ARG, "y8 is not 16-byte aligned");
  if (!(eps >= 0.f)) return operator_fail(GAN_E_ARG, "eps is negative");
  for (const gan_status s : {check_matrix(x, x_stride, cols, "x_stride is below cols"), check_matrix(residual, residual_stride, cols, "residual_stride is below cols"),
                             check_matrix(sum, sum_stride, cols, "sum_stride is below cols"), check_matrix(y, y_stride, cols, "y_stride is below cols")})
    if (s) return s;
  if (rows == 0) return GAN_OK;
  operator_launches();
  const int e = precision == GAN_FP32 ? 4 : 2;
  const bool vec = cols % E == 0 && rows_aligned16(x, x_stride, e) && (!residual || rows_aligned16(residual, residual_stride, e)) && aligned16(gain) &&
                   (!sum || rows_aligned16(sum, sum_stride, e)) && (!y || rows_aligned16(y, y_stride, e));
  const NormArgs a = {x, residual, gain, sum, y, y8, y8_scale, inv_rms, x_stride, residual_stride, sum_stride, y_stride, rows, cols, eps};
  const hipStream_t st = (hipStream_t)hip_stream;
  const auto go = [&](auto t) {
    typedef decltype(t) T;
    if (!vec) launch_norm<T, false, false>(a, st);
    else if (rows * cols * ((sum ? e : 0) + (y ? e : 0) + (y8 ? 1 : 0)) > PAST_CACHES) launch_norm<T, true, true>(a, st);
    else launch_norm<T, true, false>(a, st);
  };
  if (precision == GAN_FP32) go(float());
  else go(bf16_t());
  return operator_launched();
}

extern "C" int64_t gan_rms_norm_backward_bytes(int64_t rows, int32_t cols) {
  if (rows <= 0 || cols < 1 || rows > MOST_ROWS || cols > MOST_COLS) return 0;
  return (int64_t)back_blocks(rows, cols) * cols * (int64_t)sizeof(float);
}

extern "C" gan_status gan_rms_norm_backward(int32_t precision, const void* dy, int64_t dy_stride, const void* sum, int64_t sum_stride, const float* gain,
                                            const float* inv_rms, const void* dsum, int64_t dsum_stride, int64_t rows, int32_t cols, void* dx,
                                            int64_t dx_stride, float* dgain, void* work, int64_t work_bytes, void* hip_stream) {
  if (const gan_status s = check_sizes(precision, rows, cols)) return s;
  if ((rows > 0 && (!dy || !sum || !inv_rms || !dx)) || !gain) return operator_fail(GAN_E_ARG, "dy, sum, gain, inv_rms or dx is NULL");
  for (const gan_status s : {check_matrix(dy, dy_stride, cols, "dy_stride is below cols"), check_matrix(sum, sum_stride, cols, "sum_stride is below cols"),
                             check_matrix(dsum, dsum_stride, cols, "dsum_stride is below cols"), check_matrix(dx, dx_stride, cols, "dx_stride is below cols")})
    if (s) return s;
  if (dgain && (work_bytes < gan_rms_norm_backward_bytes(rows, cols) || (!work && rows > 0) || !aligned16(work)))
    return operator_fail(GAN_E_ARG, "work is smaller than gan_rms_norm_backward_bytes, or not 16-byte aligned");
  operator_launches();
  const hipStream_t st = (hipStream_t)hip_stream;
  const int e = precision == GAN_FP32 ? 4 : 2;
  if (rows > 0) {
    const bool vec = cols % E == 0 && rows_aligned16(dy, dy_stride, e) && rows_aligned16(sum, sum_stride, e) && (!dsum || rows_aligned16(dsum, dsum_stride, e)) &&
                     rows_aligned16(dx, dx_stride, e) && aligned16(gain);
    const NormBackArgs a = {dy, sum, dsum, gain, inv_rms, dx, dgain ? (float*)work : nullptr, dy_stride, sum_stride, dsum_stride, dx_stride, rows, cols};
    const auto go = [&](auto t) {
      typedef decltype(t) T;
      if (!vec) launch_back<T, false, false>(a, st);
      else if (rows * cols * e > PAST_CACHES) launch_back<T, true, true>(a, st);
      else launch_back<T, true, false>(a, st);
    };
    if (precision == GAN_FP32) go(float());
    else go(bf16_t());
  }
  if (dgain)
    by_launches((cols + 31) / 32, 16, [&](long long first, long long blocks) {
      hipLaunchKernelGGL(gain_sum_kernel, dim3((unsigned)blocks), dim3(1024), 0, st, (const float*)work, dgain, rows > 0 ? back_blocks(rows, cols) : 0, cols, (int)first * 32);
    });
  return operator_launched();
}

extern "C" gan_status gan_quantize8(int32_t precision, const void* x, int64_t x_stride, int64_t rows, int32_t cols, uint8_t* q, uint8_t* scale, void* hip_stream) {
  if (const gan_status s = check_sizes(precision, rows, cols)) return s;
  if (rows > 0 && (!x || !q || !scale)) return operator_fail(GAN_E_ARG, "x, q or scale is NULL");
  if (!aligned16(q)) return operator_fail(GAN_E_ARG, "q is not 16-byte aligned");
  if (const gan_status s = check_matrix(x, x_stride, cols, "x_stride is below cols")) return s;
  if (rows == 0) return GAN_OK;
  operator_launches();
  const int e = precision == GAN_FP32 ? 4 : 2;
  const bool vec = cols % E == 0 && rows_aligned16(x, x_stride, e);
  const long long want = (rows * (padded8(cols) / E) + 255) / 256;
  const dim3 grid((unsigned)(want < 8192 ? want : 8192));
  const hipStream_t st = (hipStream_t)hip_stream;
#define GAN_Q8(T, V) hipLaunchKernelGGL((quantize8_kernel<T, V>), grid, dim3(256), 0, st, (const T*)x, x_stride, rows, cols, q, scale)
  if (precision == GAN_FP32) { if (vec) GAN_Q8(float, true); else GAN_Q8(float, false); }
  else { if (vec) GAN_Q8(bf16_t, true); else GAN_Q8(bf16_t, false); }
#undef GAN_Q8
  return operator_launched();
}

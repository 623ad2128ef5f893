// Products grouped by label as they are: the calls, and which kernel each takes (group_product.h).
#include "group_product.h"

namespace gan {
namespace {

// dw = the parts, added in order
__global__ __launch_bounds__(256) void sum_parts_kernel(const float* parts, float* dw, long long n, int count) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
    float s = parts[i];
    for (int p = 1; p < count; ++p) s += parts[p * n + i];
    dw[i] = s;
  }
}

// Into how many parts the weight gradient takes an expert's rows: few tiles of long sums would leave most CUs idle.  As many as make two tiles of 128 a CU, of 256 rows at least, 64 at
// most.  us, in one part and so: one expert of 16384 rows, 512 x 512 (32 parts), fp32 543, 77, bf16 150, 38; 128 x 128 (64) 441, 37 and 157, 33; one of 1000, 256 x 256 (3) 31, 16.5 and
// 14.0, 11.6; four of 1000, 512 x 512 (3) 33, 26 and 15.6, 15.5; one of 4000, 2048 x 2048 (2) 248, 195, but in bf16, whose tiles of 256 are enough, 47, 57.  Half as many tiles: the first
// 90 and 31; twice as many: 96 and 54.  Parts of 128 rows: 256 x 256 13.0 and 11.6, but 512 x 512 of 1000 rows 32 and 20.6; of 512 rows: 31 and 14, 33.5 and 15.6.
int wgrad_parts(int groups, long long rows, int n_in, int n_out) {
  const long long blocks = wgrad_tiles(groups, n_out, n_in, 128), each = rows / std::max(1, groups);
  return (int)std::max(1ll, std::min({512 / std::max(1ll, blocks), each / 256, 64ll}));
}

}  // namespace
}  // namespace gan

using namespace gan;

extern "C" gan_status gan_group_linear(int32_t precision, const void* x, int64_t x_stride, const void* w, const int32_t* offs, int32_t groups, int64_t rows,
                                       int32_t n_in, int32_t n_out, void* y, int64_t y_stride, void* hip_stream) {
  if (const gan_status s = check(precision, x, y, w, offs, groups, rows, n_in, n_out)) return s;
  if (x_stride < n_in || y_stride < n_out) return operator_fail(GAN_E_ARG, "x_stride is below n_in, or y_stride below n_out");
  if (rows == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2;
  const LinearArgs q = {x, w, nullptr, nullptr, y, offs, x_stride, n_in, y_stride, (long long)n_in * n_out, 0, groups, (int)rows, 0, n_out, n_in, 1, 0, 0};
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool small = short_rows(x_stride, e) && short_rows(n_in, e), aligned = small && n_in % 8 == 0 && rows_aligned16(x, x_stride, e) && aligned16(w);
  const int few = few_rows(q, FORWARD, e);
  if (precision == GAN_FP32) return few && small ? launch_few<float, false, float>(q, few, st) : launch_fp32<FORWARD>(q, st);
  if (few && small) return aligned ? launch_few<bf16_t, false, bf16_t>(q, few, st) : launch_few<bf16_t, true, bf16_t>(q, few, st);
  return aligned ? launch_large<ALIGNED, FORWARD, bf16_t>(q, st) : launch_large<ANY, FORWARD, bf16_t>(q, st);
}

extern "C" gan_status gan_group_linear_dgrad(int32_t precision, const void* dy, int64_t dy_stride, const void* w, const int32_t* offs, int32_t groups, int64_t rows,
                                             int32_t n_in, int32_t n_out, void* dx, int64_t dx_stride, void* hip_stream) {
  if (const gan_status s = check(precision, dy, dx, w, offs, groups, rows, n_in, n_out)) return s;
  if (dy_stride < n_out || dx_stride < n_in) return operator_fail(GAN_E_ARG, "dy_stride is below n_out, or dx_stride below n_in");
  if (rows == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2;
  const LinearArgs q = {dy, w, nullptr, nullptr, dx, offs, dy_stride, n_in, dx_stride, (long long)n_in * n_out, 0, groups, (int)rows, 0, n_in, n_out, 1, 0, 0};
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool small = short_rows(dy_stride, e) && short_rows(n_in, e), aligned = small && n_out % 8 == 0 && n_in % 8 == 0 && rows_aligned16(dy, dy_stride, e) && aligned16(w);
  const int few = small && (long long)n_in * n_out * e < 1ll << 31 ? few_rows(q, DGRAD, e) : 0;
  if (precision == GAN_FP32) return few ? launch_few_dgrad<float, false>(q, few, st) : launch_fp32<DGRAD>(q, st);
  if (few) return aligned ? launch_few_dgrad<bf16_t, false>(q, few, st) : launch_few_dgrad<bf16_t, true>(q, few, st);
  return aligned ? launch_large<ALIGNED, DGRAD, bf16_t>(q, st) : launch_large<ANY, DGRAD, bf16_t>(q, st);
}

extern "C" int64_t gan_group_linear_wgrad_bytes(int32_t groups, int64_t rows, int32_t n_in, int32_t n_out) {
  if (groups < 1 || rows < 1 || n_in < 1 || n_out < 1) return 0;
  const int parts = wgrad_parts(groups, rows, n_in, n_out);
  return parts > 1 ? (int64_t)parts * groups * n_in * n_out * (int64_t)sizeof(float) : 0;
}

extern "C" gan_status gan_group_linear_wgrad(int32_t precision, const void* x, int64_t x_stride, const void* dy, int64_t dy_stride, const int32_t* offs,
                                             int32_t groups, int64_t rows, int32_t n_in, int32_t n_out, float* dw, void* work, int64_t work_bytes, void* hip_stream) {
  if (const gan_status s = check(precision, x, dy, dw, offs, groups, rows, n_in, n_out)) return s;
  if (x_stride < n_in || dy_stride < n_out) return operator_fail(GAN_E_ARG, "x_stride is below n_in, or dy_stride below n_out");
  const int64_t need = gan_group_linear_wgrad_bytes(groups, rows, n_in, n_out);
  if (work_bytes < need || (need > 0 && !work) || !aligned16(work)) return operator_fail(GAN_E_ARG, "work is smaller than gan_group_linear_wgrad_bytes, or not 16-byte aligned");
  if (groups == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2, parts = rows > 0 ? wgrad_parts(groups, rows, n_in, n_out) : 1;
  const long long n = (long long)groups * n_in * n_out;
  const LinearArgs q = {dy, x, nullptr, nullptr, parts > 1 ? work : dw, offs, dy_stride, x_stride, n_in, 0, (long long)n_in * n_out, groups, (int)rows, n_out, n_in, 0, parts, n, 0};
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool aligned = short_rows(x_stride, e) && short_rows(dy_stride, e) && n_in % 8 == 0 && n_out % 8 == 0 && rows_aligned16(x, x_stride, e) && rows_aligned16(dy, dy_stride, e);
  const gan_status s = precision == GAN_FP32 ? launch_fp32<WGRAD>(q, st) : aligned ? launch_large<ALIGNED, WGRAD, float>(q, st) : launch_large<ANY, WGRAD, float>(q, st);
  if (s != GAN_OK || parts == 1) return s;
  hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)std::min(ceil_div(n, 256), 4096ll)), dim3(256), 0, st, (const float*)work, dw, n, parts);
  return operator_launched();
}

extern "C" gan_status gan_group_linear8(const uint8_t* x8, const uint8_t* x_scale, const uint8_t* w8, const uint8_t* w_scale, const int32_t* offs, int32_t groups,
                                        int64_t rows, int32_t n_in, int32_t n_out, int32_t y_precision, void* y, int64_t y_stride, void* hip_stream) {
  if (const gan_status s = check(y_precision, x8, y, w8, offs, groups, rows, n_in, n_out)) return s;
  if ((rows > 0 && !x_scale) || (groups > 0 && !w_scale)) return operator_fail(GAN_E_ARG, "x_scale or w_scale is NULL");
  if (!aligned16(x8) || !aligned16(w8)) return operator_fail(GAN_E_ARG, "x8 or w8 is not 16-byte aligned");
  if (y_stride < n_out) return operator_fail(GAN_E_ARG, "y_stride is below n_out");
  const long long k = padded8(n_in);
  if (!short_rows(k, 1)) return operator_fail(GAN_E_SHAPE, "more than 2^22 inputs in 8 bits");
  if (rows == 0) return GAN_OK;
  const LinearArgs q = {x8, w8, x_scale, w_scale, y, offs, k, k, y_stride, k * n_out, 0, groups, (int)rows, 0, n_out, (int)k, 1, 0, 0};
  const hipStream_t st = (hipStream_t)hip_stream;
  if (const int few = few_rows(q, FORWARD, 1))
    return y_precision == GAN_FP32 ? launch_few<uint8_t, false, float>(q, few, st) : launch_few<uint8_t, false, bf16_t>(q, few, st);
  return y_precision == GAN_FP32 ? launch_large<EIGHT_BITS, FORWARD, float>(q, st) : launch_large<EIGHT_BITS, FORWARD, bf16_t>(q, st);
}

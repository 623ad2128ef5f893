// Products grouped by label with bias, activation and residual in their epilogue, and the gradient that goes through the activation before them: the calls, and which kernel
// each takes (group_product.h, whose rules are those of the products without but where they say so).
#include "group_product.h"

using namespace gan;

namespace {

gan_status check_epilogue(int32_t act, const void* add, long long add_stride, const void* z, long long z_stride, int32_t cols, const char* add_why) {
  if (!act_known(act)) return operator_fail(GAN_E_ARG, "unknown activation");
  if (add && add_stride < cols) return operator_fail(GAN_E_ARG, add_why);
  if (z && z_stride < cols) return operator_fail(GAN_E_ARG, "z_stride is below the row's length");
  return GAN_OK;
}

// Sixteens of rows for the kernel for few rows in 8 bits.  Next to few_rows(): experts of up to 64 rows go to tiles, two sets of waves to each, where those are at most one a CU while this kernel's
// blocks, each of which converts all of its codes, are several turns of a long sum (us by this kernel, in tiles): four experts of 32, 4096 -> 4096: 46, 32; eight of 32, 4096 -> 2048: 51, 32; eight of
// 16, 4096 -> 4096: 54, 37; 16 of 25, 2048 -> 1280: 20.3, 19.1; but eight of 50, 2048 -> 1024: 15, 18; one of 64, 4096 -> 4096: 19, 28; 16 of 12, 2048 -> 2432 (304 tiles): 29, 37; one of 160,
// 4096 -> 2816: 32, 39; two of 60, 8192 -> 2048: 50, 68.
int few_rows8(const LinearArgs& q) {
  const int few = few_rows(q, FORWARD, 1);
  const long long groups = most_groups(q), each = q.rows / groups;
  const bool tiled = each <= 64 && q.k <= 4096 && groups * ceil_div(q.n, 128) <= 256 && (q.rows + 16 * groups) * ceil_div(q.n, 32) * q.k > 50ll << 20;
  return few == 2 && tiled ? 0 : few;
}

}  // namespace

extern "C" gan_status gan_group_linear_act(int32_t precision, const void* x, int64_t x_stride, const void* w, const int32_t* offs, int32_t groups, int64_t rows, int32_t n_in,
                                           int32_t n_out, const float* bias, int32_t act, const void* residual, int64_t residual_stride, void* z, int64_t z_stride, void* y,
                                           int64_t y_stride, void* hip_stream) {
  if (const gan_status s = check(precision, x, y, w, offs, groups, rows, n_in, n_out)) return s;
  if (const gan_status s = check_epilogue(act, residual, residual_stride, z, z_stride, n_out, "residual_stride is below n_out")) return s;
  if (x_stride < n_in || y_stride < n_out) return operator_fail(GAN_E_ARG, "x_stride is below n_in, or y_stride below n_out");
  if (rows == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2;
  const LinearArgs p = {x, w, nullptr, nullptr, y, offs, x_stride, n_in, y_stride, (long long)n_in * n_out, 0, groups, (int)rows, 0, n_out, n_in, 1, 0, 0};
  const ActArgs q = {p, bias, residual, nullptr, z, residual_stride, z_stride, act};
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool small = short_rows(x_stride, e) && short_rows(n_in, e), aligned = small && n_in % 8 == 0 && rows_aligned16(x, x_stride, e) && aligned16(w);
  const int few = few_rows(q, FORWARD, e);
  if (precision == GAN_FP32) return few && small ? launch_few<float, false, float>(q, few, st) : launch_fp32<FORWARD>(q, st);
  if (few && small) return aligned ? launch_few<bf16_t, false, bf16_t>(q, few, st) : launch_few<bf16_t, true, bf16_t>(q, few, st);
  return aligned ? launch_large<ALIGNED, FORWARD, bf16_t>(q, st) : launch_large<ANY, FORWARD, bf16_t>(q, st);
}

extern "C" gan_status gan_group_linear_dgrad_act(int32_t precision, const void* dy, int64_t dy_stride, const void* w, const int32_t* offs, int32_t groups, int64_t rows,
                                                 int32_t n_in, int32_t n_out, const void* other, int64_t other_stride, int32_t act, const void* z, int64_t z_stride, void* dx,
                                                 int64_t dx_stride, void* hip_stream) {
  if (const gan_status s = check(precision, dy, dx, w, offs, groups, rows, n_in, n_out)) return s;
  if (const gan_status s = check_epilogue(act, other, other_stride, act != GAN_ACT_NONE ? z : nullptr, z_stride, n_in, "other_stride is below n_in")) return s;
  if (rows > 0 && act != GAN_ACT_NONE && !z) return operator_fail(GAN_E_ARG, "z is NULL");
  if (dy_stride < n_out || dx_stride < n_in) return operator_fail(GAN_E_ARG, "dy_stride is below n_out, or dx_stride below n_in");
  if (rows == 0) return GAN_OK;
  const int e = precision == GAN_FP32 ? 4 : 2;
  const LinearArgs p = {dy, w, nullptr, nullptr, dx, offs, dy_stride, n_in, dx_stride, (long long)n_in * n_out, 0, groups, (int)rows, 0, n_in, n_out, 1, 0, 0};
  const ActArgs q = {p, nullptr, other, z, nullptr, other_stride, z_stride, act};
  const hipStream_t st = (hipStream_t)hip_stream;
  const bool small = short_rows(dy_stride, e) && short_rows(n_in, e), aligned = small && n_out % 8 == 0 && n_in % 8 == 0 && rows_aligned16(dy, dy_stride, e) && aligned16(w);
  const int few = small && (long long)n_in * n_out * e < 1ll << 31 ? few_rows(q, DGRAD, e) : 0;
  if (precision == GAN_FP32) return few ? launch_few_dgrad<float, false>(q, few, st) : launch_fp32<DGRAD>(q, st);
  if (few) return aligned ? launch_few_dgrad<bf16_t, false>(q, few, st) : launch_few_dgrad<bf16_t, true>(q, few, st);
  return aligned ? launch_large<ALIGNED, DGRAD, bf16_t>(q, st) : launch_large<ANY, DGRAD, bf16_t>(q, st);
}

extern "C" gan_status gan_group_linear8_act(const uint8_t* x8, const uint8_t* x_scale, const uint8_t* w8, const uint8_t* w_scale, const int32_t* offs, int32_t groups,
                                            int64_t rows, int32_t n_in, int32_t n_out, const float* bias, int32_t act, const void* residual, int64_t residual_stride,
                                            int32_t y_precision, void* y, int64_t y_stride, void* hip_stream) {
  if (const gan_status s = check(y_precision, x8, y, w8, offs, groups, rows, n_in, n_out)) return s;
  if ((rows > 0 && !x_scale) || (groups > 0 && !w_scale)) return operator_fail(GAN_E_ARG, "x_scale or w_scale is NULL");
  if (!aligned16(x8) || !aligned16(w8)) return operator_fail(GAN_E_ARG, "x8 or w8 is not 16-byte aligned");
  if (const gan_status s = check_epilogue(act, residual, residual_stride, nullptr, 0, n_out, "residual_stride is below n_out")) return s;
  if (y_stride < n_out) return operator_fail(GAN_E_ARG, "y_stride is below n_out");
  const long long k = padded8(n_in);
  if (!short_rows(k, 1)) return operator_fail(GAN_E_SHAPE, "more than 2^22 inputs in 8 bits");
  if (rows == 0) return GAN_OK;
  const LinearArgs p = {x8, w8, x_scale, w_scale, y, offs, k, k, y_stride, k * n_out, 0, groups, (int)rows, 0, n_out, (int)k, 1, 0, 0};
  const ActArgs q = {p, bias, residual, nullptr, nullptr, residual_stride, 0, act};
  const hipStream_t st = (hipStream_t)hip_stream;
  if (const int few = few_rows8(q))
    return y_precision == GAN_FP32 ? launch_few<uint8_t, false, float>(q, few, st) : launch_few<uint8_t, false, bf16_t>(q, few, st);
  return y_precision == GAN_FP32 ? launch_large<EIGHT_BITS, FORWARD, float>(q, st) : launch_large<EIGHT_BITS, FORWARD, bf16_t>(q, st);
}

// Texts of the operators' refusals, one for each thread, and the checks that they share.
#include "operators.h"

namespace gan {
namespace {
thread_local const char* g_why = "";
}

gan_status operator_fail(gan_status s, const char* why) {
  g_why = why;
  return s;
}

gan_status check_matrix(const void* p, long long stride, int cols, const char* why) {
  return p && stride < cols ? operator_fail(GAN_E_ARG, why) : GAN_OK;
}
gan_status check_sizes(int32_t precision, long long rows, int cols) {
  if (precision != GAN_FP32 && precision != GAN_BF16_FP32MASTER) return operator_fail(GAN_E_ARG, "unknown precision");
  if (rows < 0 || cols < 1) return operator_fail(GAN_E_ARG, "negative rows or no columns");
  if (rows > MOST_ROWS || cols > MOST_COLS) return operator_fail(GAN_E_SHAPE, "more than 2^30 rows or 2^28 columns");
  return GAN_OK;
}

void operator_launches() { (void)hipGetLastError(); }

gan_status operator_launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GAN_OK : operator_fail(GAN_E_HIP, hipGetErrorString(e));
}

}  // namespace gan

extern "C" const char* gan_operator_last_error(void) { return gan::g_why; }

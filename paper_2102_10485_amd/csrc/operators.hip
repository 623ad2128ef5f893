// Texts of the operators' refusals, one for each thread.
#include "operators.h"

namespace gan {
namespace {
thread_local const char* g_why = "";
}

gan_status operator_fail(gan_status s, const char* why) {
  g_why = why;
  return s;
}

void operator_launches() { (void)hipGetLastError(); }

gan_status operator_launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GAN_OK : operator_fail(GAN_E_HIP, hipGetErrorString(e));
}

}  // namespace gan

extern "C" const char* gan_operator_last_error(void) { return gan::g_why; }

// What an 8-bit operand of the grouped products asks for, walked on the host (tests/test_code_walk.py).
#include "../../paper_2102_10485_amd/csrc/code_walk.h"

extern "C" void code_walk(int k0, int k_end, int writes, int* asked) {
  gan::CodeWalk w;
  w.start(k0);
  *asked++ = w.k;                                    // before the first step is written
  w.started(k_end);
  int left = k_end - k0;
  for (int i = 0; i < writes; ++i, left -= gan::CODE_STEP) {
    *asked++ = w.k;
    w.asked(left);
  }
}
